"""What training with a policy, learning from a teacher and a layer with a matrix for its memory give this library, as cases to be timed.

Three operators.  `logprobs`: the log-probability of a given token per row of logits, the entropy of the row and its best
alternatives - an action's in a knob, a token's of a vocabulary - and the gradient by the logits.  `distill`: the divergence of a
row's distribution from a teacher's best entries, which is what the first one lists, and its gradient.  `delta`: the gated delta
rule, a recurrence whose state is a matrix per head, S_t = exp(g_t) S_{t-1} + beta_t k_t (v_t - exp(g_t) S_{t-1}^T k_t)^T, read as
o_t = scale S_t^T q_t, with its backward pass and its step for single tokens.

Where `own` is false a pass is made of elementary torch operations in 32 bits (sums of log-decays in 64); where it is true it is
the library's call.  Alternatives are ordered by descending logit, equal ones by ascending index.
"""
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CHUNK = 64                                               # steps that the plain form of the delta rule takes together


def listed():
    return [
        # an ordinary trajectory's actions (65,536 configurations, 8 knobs, 3 directions), some steps padded: the forward pass of an epoch
        {"name": "logprobs_actions", "kind": "logprobs", "rows": 524288, "v": 3, "type": "f32", "temperature": 0, "top": 0, "backward": 0, "masked": 0},
        # and its backward pass, with an entropy bonus
        {"name": "logprobs_actions_back", "kind": "logprobs", "rows": 524288, "v": 3, "type": "f32", "temperature": 0, "top": 0, "backward": 1, "masked": 0},
        # a few choices out of a small trajectory's scores, with their best alternatives: latency
        {"name": "logprobs_small", "kind": "logprobs", "rows": 8, "v": 2000, "type": "f32", "temperature": 1, "top": 5, "backward": 0, "masked": 0},
        # a serving batch over a vocabulary, with alternatives and a temperature per request, some entries not allowed
        {"name": "logprobs_vocab", "kind": "logprobs", "rows": 64, "v": 128003, "type": "bf16", "temperature": 1, "top": 20, "backward": 0, "masked": 1},
        # a training batch over a vocabulary: gradients
        {"name": "logprobs_train", "kind": "logprobs", "rows": 8192, "v": 32001, "type": "bf16", "temperature": 0, "top": 0, "backward": 1, "masked": 0},
        # a small student over few choices: latency
        {"name": "distill_small", "kind": "distill", "rows": 256, "v": 1000, "k": 8, "type": "f32", "temperature": 1, "backward": 0},
        # a training batch over a vocabulary and the 32 best entries of its teacher
        {"name": "distill_vocab", "kind": "distill", "rows": 4096, "v": 50021, "k": 32, "type": "bf16", "temperature": 1, "backward": 0},
        # a larger vocabulary and 64 entries: gradients
        {"name": "distill_train", "kind": "distill", "rows": 2048, "v": 128003, "k": 64, "type": "bf16", "temperature": 1, "backward": 1},
        # one token of a layer in serving, 64 sequences
        {"name": "delta_step", "kind": "delta", "batch": 64, "t": 1, "heads": 32, "key_heads": 16, "dk": 128, "dv": 128, "type": "bf16", "reset": 0, "backward": 0},
        # the steps of a few short episodes in a small layer: latency
        {"name": "delta_small", "kind": "delta", "batch": 4, "t": 37, "heads": 4, "key_heads": 4, "dk": 64, "dv": 64, "type": "f32", "reset": 1, "backward": 0},
        # a long prompt, heads sharing keys
        {"name": "delta_prompt", "kind": "delta", "batch": 1, "t": 8191, "heads": 32, "key_heads": 16, "dk": 128, "dv": 128, "type": "bf16", "reset": 0, "backward": 0},
        # the backward pass of a layer in training, sequences packed behind each other
        {"name": "delta_train", "kind": "delta", "batch": 4, "t": 2048, "heads": 16, "key_heads": 16, "dk": 128, "dv": 128, "type": "bf16", "reset": 1, "backward": 1},
    ]


def _between(rng, lo, hi):
    """A whole number in lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """Another case: any of the three, sizes between the smallest and the largest listed."""
    kind = rng.choice(["logprobs", "distill", "delta"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    backward = rng.randint(0, 1)
    if kind == "delta":
        heads = rng.choice([1, 2, 4, 6, 8, 16, 32])
        case = {"kind": kind, "heads": heads, "key_heads": rng.choice([h for h in (1, 2, 3, 4, 8, 16, 32) if heads % h == 0]),
                "dk": _between(rng, 16, 128), "dv": _between(rng, 16, 128), "type": dtype, "reset": rng.randint(0, 1), "backward": backward}
        case["t"] = rng.choice([1, _between(rng, 2, 8191), _between(rng, 64, 8191)])
        room = (1 << (31 if backward else 32)) // (heads * case["dk"] * case["dv"])        # tokens
        case["t"] = min(case["t"], room)
        case["batch"] = _between(rng, 1, min(64, room // case["t"]))
        return case
    case = {"kind": kind, "v": _between(rng, 3 if kind == "logprobs" else 16, 128003), "type": dtype, "temperature": rng.randint(0, 1), "backward": backward}
    if kind == "logprobs":
        case["top"] = 0 if backward or case["v"] < 16 else rng.choice([0, rng.randint(1, 8), rng.randint(8, 64)])
        case["top"] = min(case["top"], case["v"] // 4)
        case["masked"] = rng.randint(0, 1) if case["v"] >= 64 else 0
        room = (1 << (25 if case["top"] else 27)) // case["v"]
    else:
        case["k"] = _between(rng, 1, min(128, case["v"] // 2))
        room = (1 << 27) // case["v"]
    case["rows"] = _between(rng, 1, min(524288, max(1, room)))
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")        # noqa: E731
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")      # noqa: E731
    s = {"case": case}
    if case["kind"] == "delta":
        return _prepare_delta(s, case, rand, randn)
    rows, v, dtype = case["rows"], case["v"], _TYPES[case["type"]]
    x = randn(rows, v).mul_(2.0).to(dtype)
    s["temperature"] = 0.5 + rand(rows) if case["temperature"] else None
    if case["kind"] == "logprobs":
        token = (rand(rows) * v).long().clamp_(max=v - 1)
        if case["masked"]:
            allowed = x.gather(1, token[:, None])
            x.masked_fill_(rand(rows, v) < 0.1, -torch.inf)
            x.scatter_(1, token[:, None], allowed)
        token = token.to(torch.int32)
        if rows >= 1024:                                 # padded steps
            token.masked_fill_(rand(rows) < 0.02, -1)
        s["logits"], s["token"] = x, token
        if case["backward"]:
            s["dlogprob"], s["dentropy"] = randn(rows), -0.1 * rand(rows)
            s["norm"], s["entropy"] = _norm(x, s["temperature"])
    else:
        s["logits"] = x
        # the teacher: its best entries come with scores that fall, a few of them beside the student's own
        k = case["k"]
        first = (rand(rows, 1) * v).long()
        step = 1 + (rand(rows, 1) * ((v - 1) // k)).long()
        s["teacher_tokens"] = ((first + step * torch.arange(k, device="cuda")) % v).to(torch.int32)
        s["teacher_logits"] = (randn(rows, k) * 0.5 - 3.0 * torch.arange(k, device="cuda") / k).to(dtype)
        if case["backward"]:
            s["dloss"] = rand(rows) / rows
            s["norm"], _ = _norm(x, s["temperature"])
    if own and not case["backward"]:                     # scratch memory, as a program's loop keeps it
        from paper_1905_12799_amd import binding as rls
        need = rls.token_logprobs_workspace_bytes(rows, v, case["top"]) if case["kind"] == "logprobs" else rls.distill_loss_workspace_bytes(rows, v)
        s["workspace"] = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    return s


def _prepare_delta(s, case, rand, randn):
    b, t, h, hk, dk, dv, dtype = (case[x] for x in ("batch", "t", "heads", "key_heads", "dk", "dv", "type"))
    dtype = _TYPES[dtype]
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)                              # noqa: E731
    s["q"], s["k"] = unit(randn(b, t, hk, dk)).to(dtype), unit(randn(b, t, hk, dk)).to(dtype)
    s["v"] = randn(b, t, h, dv).to(dtype)
    s["g"] = -torch.nn.functional.softplus(1.5 * randn(b, t, h) - 3.0)
    s["beta"] = torch.sigmoid(randn(b, t, h))
    s["state"] = 0.1 * randn(b, h, dk, dv)
    s["reset"] = (rand(b, t) < 1.0 / 300).to(torch.uint8) if case["reset"] else None
    if case["backward"]:
        s["do"] = randn(b, t, h, dv).to(dtype)
        s["dlast"] = 0.1 * randn(b, h, dk, dv)
    if own:
        from paper_1905_12799_amd import binding as rls
        need = rls.gated_delta_workspace_bytes(b, t, h, hk, dk, dv, backward=bool(case["backward"]))
        s["workspace"] = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    return {"logprobs": _run_logprobs, "distill": _run_distill, "delta": _run_delta}[s["case"]["kind"]](s)


def _run_logprobs(s):
    case, x = s["case"], s["logits"]
    if own:
        from paper_1905_12799_amd import binding as rls
        if case["backward"]:
            return {"dlogits": rls.token_logprobs_backward(x, s["token"], s["norm"], s["entropy"], s["dlogprob"], s["dentropy"], temperature=s["temperature"])}
        r = rls.token_logprobs(x, s["token"], temperature=s["temperature"], top=case["top"], workspace=s["workspace"])
        out = {"logprob": r.logprob, "entropy": r.entropy}
        if case["top"]:
            out["top_logprob"], out["top_token"] = r.top_logprob, r.top_token
        return out
    token = s["token"].long()[:, None]
    given = (token >= 0) & (token < case["v"])
    token = token.clamp(0, case["v"] - 1)
    if case["backward"]:
        logp = _distances(x, s["norm"][:, :1], s["temperature"]) - s["norm"][:, 1:]
        p = torch.exp(logp)
        dlogprob = torch.where(given, s["dlogprob"][:, None], 0.0)
        d = -p * (dlogprob + s["dentropy"][:, None] * (torch.where(p > 0, logp, 0.0) + s["entropy"][:, None]))
        d.scatter_add_(1, token, dlogprob)
        if s["temperature"] is not None:
            d *= (1.0 / s["temperature"])[:, None]
        return {"dlogits": d.masked_fill_(x == -torch.inf, 0.0).to(x.dtype)}
    norm, entropy = _norm(x, s["temperature"])
    logp = _distances(x, norm[:, :1], s["temperature"]) - norm[:, 1:]
    out = {"logprob": torch.where(given, logp.gather(1, token), 0.0)[:, 0], "entropy": entropy}
    if case["top"]:
        best = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
        out["top_logprob"], out["top_token"] = logp.gather(1, best), best.to(torch.int32)
    return out


def _distances(x, top, temperature):
    """(x - largest) / temperature in 32 bits."""
    d = x.float() - top
    return d if temperature is None else d * (1.0 / temperature)[:, None]


def _norm(x, temperature):
    """Of every row the largest logit and log(sum(exp(d))) side by side, and the entropy."""
    top = x.float().amax(1, keepdim=True)
    d = _distances(x, top, temperature)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log = torch.log(total)
    entropy = log - (torch.where(e > 0, d, 0.0) * e).sum(1, keepdim=True) / total
    return torch.cat([top, log], 1), entropy[:, 0]


def _run_distill(s):
    case, x, tokens, logits = s["case"], s["logits"], s["teacher_tokens"], s["teacher_logits"]
    if own:
        from paper_1905_12799_amd import binding as rls
        if case["backward"]:
            return {"dlogits": rls.distill_loss_backward(x, tokens, logits, s["norm"], s["dloss"], temperature=s["temperature"])}
        return {"loss": rls.distill_loss(x, tokens, logits, temperature=s["temperature"], workspace=s["workspace"])[0]}
    d = _distances(logits, logits.float().amax(1, keepdim=True), s["temperature"])
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    p = e / total
    if case["backward"]:
        q = torch.exp(_distances(x, s["norm"][:, :1], s["temperature"]) - s["norm"][:, 1:])
        q.scatter_add_(1, tokens.long(), -p)
        scale = s["dloss"] if s["temperature"] is None else s["dloss"] / s["temperature"]
        return {"dlogits": (q * scale[:, None]).to(x.dtype)}
    norm, _ = _norm(x, s["temperature"])
    logq = _distances(x.gather(1, tokens.long()), norm[:, :1], s["temperature"]) - norm[:, 1:]
    return {"loss": (p * ((d - torch.log(total)) - logq)).sum(1)}


def _run_delta(s):
    if own:
        from paper_1905_12799_amd import binding as rls
        if s["case"]["backward"]:
            names = ("dq", "dk", "dv", "dg", "dbeta", "dstate")
            return dict(zip(names, rls.gated_delta_backward(s["q"], s["k"], s["v"], s["g"], s["beta"], s["do"], state=s["state"], reset=s["reset"],
                                                            dlast=s["dlast"], workspace=s["workspace"])))
        o, last = rls.gated_delta(s["q"], s["k"], s["v"], s["g"], s["beta"], state=s["state"], reset=s["reset"], workspace=s["workspace"])
        return {"o": o, "last": last}
    c = _chunks(s)
    before, y, last = _forward(c, s["state"])
    if s["case"]["backward"]:
        return _backward(c, s, before, y)
    o = c["scale"] * (c["a"][..., None] * (c["q"] @ before) + c["p"] @ (c["beta"][..., None] * y))
    return {"o": _steps(o, s["case"]).to(s["v"].dtype), "last": last}


def _chunks(s):
    """The steps in chunks [batch, heads, chunks, CHUNK, ...] with what their products need, all in 32 bits."""
    case = s["case"]
    b, t, h, hk, dk = (case[x] for x in ("batch", "t", "heads", "key_heads", "dk"))
    n = -(-t // CHUNK)

    def cut(x):                                          # [batch, steps, heads, ...], zeros behind the last step
        x = torch.cat([x, torch.zeros(b, n * CHUNK - t, *x.shape[2:], dtype=x.dtype, device=x.device)], 1)
        return x.view(b, n, CHUNK, *x.shape[2:]).movedim(3, 1).contiguous()
    shared = lambda x: cut(x.float().repeat_interleave(h // hk, 2))                # noqa: E731
    c = {"q": shared(s["q"]), "k": shared(s["k"]), "v": cut(s["v"].float()), "beta": cut(s["beta"]), "scale": dk ** -0.5}
    reset = torch.zeros(b, t, dtype=torch.uint8, device="cuda") if s["reset"] is None else s["reset"]
    c["cut"] = cut(reset[:, :, None].expand(b, t, h)) != 0
    part = c["cut"].long().cumsum(-1)
    gamma = torch.where(c["cut"], 0.0, cut(s["g"])).double().cumsum(-1)
    same = (part[..., :, None] == part[..., None, :]).tril()
    decay = torch.where(same, torch.exp((gamma[..., :, None] - gamma[..., None, :]).clamp(max=0.0).float()), 0.0)
    c["decay"] = decay
    c["a"] = torch.where(part == 0, torch.exp(gamma.float()), 0.0)                 # what is left of the state before the chunk
    c["c"] = decay[..., -1, :]                                                     # and of a step behind it
    c["kk"] = (decay * (c["k"] @ c["k"].transpose(-1, -2))).tril(-1)
    c["p"] = decay * (c["q"] @ c["k"].transpose(-1, -2))
    m = c["kk"] * c["beta"][..., None, :]
    inv = torch.eye(CHUNK, device="cuda").expand_as(m).contiguous()
    for i in range(1, CHUNK):                            # (1 + m) inv = 1, row by row
        inv[..., i:i + 1, :] -= m[..., i:i + 1, :i] @ inv[..., :i, :]
    c["inv"] = inv
    return c


def _forward(c, state):
    """The state before every chunk, y_t = v_t - (decayed state)^T k_t of every step, and the state after the last."""
    y0 = c["inv"] @ c["v"]
    w = c["inv"] @ (c["a"][..., None] * c["k"])
    kept = ((c["c"] * c["beta"])[..., None] * c["k"]).transpose(-1, -2)
    before, ys = [], []
    for i in range(c["v"].shape[2]):
        before.append(state)
        y = y0[:, :, i] - w[:, :, i] @ state
        ys.append(y)
        state = c["a"][:, :, i, -1, None, None] * state + kept[:, :, i] @ y
    return torch.stack(before, 2), torch.stack(ys, 2), state


def _steps(x, case):
    """[batch, heads, chunks, CHUNK, ...] as [batch, steps, heads, ...]."""
    return x.movedim(1, 3).flatten(1, 2)[:, :case["t"]].contiguous()


def _backward(c, s, before, y):
    case, scale = s["case"], c["scale"]
    b, t, h, hk = (case[x] for x in ("batch", "t", "heads", "key_heads"))
    n = y.shape[2]
    do = torch.cat([s["do"].float(), torch.zeros(b, n * CHUNK - t, h, case["dv"], device="cuda")], 1)
    do = do.view(b, n, CHUNK, h, case["dv"]).movedim(3, 1).contiguous()
    q, k, a, beta = c["q"], c["k"], c["a"][..., None], c["beta"][..., None]
    turned = c["inv"].transpose(-1, -2)
    e = turned @ (beta * (scale * (c["p"].transpose(-1, -2) @ do)))
    f = turned @ (beta * c["c"][..., None] * k)
    direct = scale * ((a * q).transpose(-1, -2) @ do)
    back = (a * k).transpose(-1, -2)
    dstate, after, dys = s["dlast"], [], []
    for i in reversed(range(n)):
        after.append(dstate)
        dy = e[:, :, i] + f[:, :, i] @ dstate
        dys.append(dy)
        dstate = c["a"][:, :, i, -1, None, None] * dstate + direct[:, :, i] - back[:, :, i] @ dy
    after, dy = torch.stack(after[::-1], 2), torch.stack(dys[::-1], 2)
    u = beta * y
    from_o, from_y = do @ y.transpose(-1, -2), dy @ y.transpose(-1, -2)            # do_i . y_j, dy_i . y_j
    by_p, by_kk = scale * c["p"] * from_o, c["kk"] * from_y
    decay = c["decay"]
    dqk = scale * from_o * beta.transpose(-1, -2) * decay
    dkk = (-from_y * beta.transpose(-1, -2) * decay).tril(-1)
    o_state = scale * a * (do @ before.transpose(-1, -2))
    y_state = a * (dy @ before.transpose(-1, -2))
    carried = c["c"][..., None] * (y @ after.transpose(-1, -2))
    dq = o_state + dqk @ k
    dk = dqk.transpose(-1, -2) @ q + dkk @ k + dkk.transpose(-1, -2) @ k + beta * carried - y_state
    kept = (k * carried).sum(-1)
    dbeta = (by_p - by_kk).sum(-2) + kept
    dgamma = (q * o_state).sum(-1) - (k * y_state).sum(-1) + ((by_p - by_kk) * beta.transpose(-1, -2)).sum(-1) - c["beta"] * dbeta
    dgamma[..., -1] += (c["beta"] * kept).sum(-1) + c["a"][..., -1] * (before * after).sum((-1, -2))
    dg = dgamma.double().flip(-1).cumsum(-1).flip(-1).float().masked_fill(c["cut"], 0.0)
    group = lambda x: _steps(x, case).unflatten(2, (hk, h // hk)).sum(3).to(s["q"].dtype)      # noqa: E731
    return {"dq": group(dq), "dk": group(dk), "dv": _steps(dy, case).to(s["v"].dtype), "dg": _steps(dg, case), "dbeta": _steps(dbeta, case), "dstate": dstate}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    """Inputs read once, outputs written once.  Per logit a subtraction, an exponential and two sums, and as many for a gradient; per token
    and head of the delta rule seven operations per entry of the state (decay, two products with it, an update), twenty with gradients."""
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}[case["type"]]
    if case["kind"] == "delta":
        tokens = float(case["batch"]) * case["t"]
        qk, v = tokens * case["key_heads"] * case["dk"] * size, tokens * case["heads"] * case["dv"] * size
        gates = tokens * case["heads"] * 8.0
        flags = tokens if case["reset"] else 0.0
        entries = float(case["heads"]) * case["dk"] * case["dv"]
        state = 8.0 * case["batch"] * entries
        if case["backward"]:
            return {"bytes": 4 * qk + 3 * v + 2 * gates + flags + 1.5 * state, "flops": 20.0 * tokens * entries}
        return {"bytes": 2 * qk + 2 * v + gates + flags + state, "flops": 7.0 * tokens * entries}
    rows, n = float(case["rows"]), float(case["rows"]) * case["v"]
    bytes_ = n * size * (2 if case["backward"] else 1) + (4.0 * rows if case["temperature"] else 0.0)
    if case["kind"] == "logprobs":
        bytes_ += rows * (24.0 if case["backward"] else 12.0 + 8.0 * case["top"])
    else:
        bytes_ += rows * (case["k"] * (4.0 + size) + (12.0 if case["backward"] else 4.0))
    return {"bytes": bytes_, "flops": 5.0 * n}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "distill": _exact_distill, "delta": _exact_delta}[case["kind"]](s)


def _parts(rows, v):
    """Rows taken together, so that their 64-bit copies stay below a gigabyte."""
    size = max(1, (1 << 27) // v)
    return [slice(i, min(i + size, rows)) for i in range(0, rows, size)]


def _scaled(s, part):
    x = s["logits"][part].double()
    return x if s["temperature"] is None else x / s["temperature"][part].double()[:, None]


def _exact_logprobs(s):
    case = s["case"]
    done = []
    for part in _parts(case["rows"], case["v"]):
        logp = torch.log_softmax(_scaled(s, part), 1)
        p = logp.exp()
        plogp = torch.where(p > 0, p * logp, 0.0)
        token = s["token"][part].long()
        given = token >= 0
        here = torch.nn.functional.one_hot(token.clamp(min=0), case["v"]).bool() if case["v"] <= 64 else None
        entropy = -plogp.sum(1)
        if case["backward"]:
            t = 1.0 if s["temperature"] is None else s["temperature"][part].double()[:, None]
            by_token = s["dlogprob"][part].double()[:, None] * given[:, None]
            d = -by_token * p - s["dentropy"][part].double()[:, None] * (plogp + p * entropy[:, None])
            if here is not None:
                d += by_token * here
            else:
                d[torch.arange(len(token), device="cuda"), token.clamp(min=0)] += by_token[:, 0]
            done.append({"dlogits": torch.where(s["logits"][part] == -torch.inf, 0.0, d / t)})
            continue
        out = {"logprob": torch.where(given, logp.gather(1, token.clamp(min=0)[:, None])[:, 0], 0.0), "entropy": entropy}
        if case["top"]:
            x = s["logits"][part].double()
            best = torch.argsort(-x, dim=1, stable=True)[:, :case["top"]]
            out["top_logprob"], out["top_token"] = logp.gather(1, best), best.to(torch.int32)
        done.append(out)
    return {name: torch.cat([d[name] for d in done]) for name in done[0]}


def _exact_distill(s):
    case = s["case"]
    done = []
    for part in _parts(case["rows"], case["v"]):
        logq = torch.log_softmax(_scaled(s, part), 1)
        t = 1.0 if s["temperature"] is None else s["temperature"][part].double()[:, None]
        logp = torch.log_softmax(s["teacher_logits"][part].double() / t, 1)
        tokens = s["teacher_tokens"][part].long()
        if case["backward"]:
            target = torch.zeros_like(logq).scatter_add_(1, tokens, logp.exp())
            done.append({"dlogits": (logq.exp() - target) * (s["dloss"][part].double()[:, None] / t)})
        else:
            done.append({"loss": (logp.exp() * (logp - logq.gather(1, tokens))).sum(1)})
    return {name: torch.cat([d[name] for d in done]) for name in done[0]}


def _exact_delta(s):
    """Step by step, the state before every step kept for the way back."""
    case = s["case"]
    b, t, h, hk, dk, dv = (case[x] for x in ("batch", "t", "heads", "key_heads", "dk", "dv"))
    if case["backward"] and 8.0 * b * t * h * dk * dv > 48e9 or 1e-4 * t + 3e-11 * b * t * h * dk * dv > 18:
        return None
    wide = lambda x: x.double().repeat_interleave(h // hk, 2)                      # noqa: E731
    q, k, v, scale = wide(s["q"]), wide(s["k"]), s["v"].double(), float(dk) ** -0.5
    carry, beta = torch.exp(s["g"].double()), s["beta"].double()
    if s["reset"] is not None:
        carry = carry * (s["reset"] == 0)[:, :, None]
    state, o, kept = s["state"].double(), torch.empty_like(v), []
    for i in range(t):
        kept.append(state) if case["backward"] else None
        state = state * carry[:, i, :, None, None]
        y = v[:, i] - (state * k[:, i, :, :, None]).sum(2)
        state = state + k[:, i, :, :, None] * (beta[:, i, :, None] * y)[:, :, None]
        o[:, i] = scale * (state * q[:, i, :, :, None]).sum(2)
    if not case["backward"]:
        return {"o": o, "last": state}
    do, ds = s["do"].double(), s["dlast"].double()
    dq, dk_, dv_, dg, dbeta = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(carry), torch.empty_like(beta)
    for i in reversed(range(t)):
        old = kept.pop() * carry[:, i, :, None, None]
        ki, bi = k[:, i, :, :, None], beta[:, i, :, None]
        y = v[:, i] - (old * ki).sum(2)
        new = old + ki * (bi * y)[:, :, None]
        ds = ds + scale * q[:, i, :, :, None] * do[:, i, :, None]
        dq[:, i] = scale * (new * do[:, i, :, None]).sum(3)
        back = (ds * ki).sum(2)                          # the gradient by beta y
        dbeta[:, i] = (back * y).sum(2)
        dy = bi * back
        dk_[:, i] = (ds * (bi * y)[:, :, None]).sum(3) - (old * dy[:, :, None]).sum(3)
        dv_[:, i] = dy
        ds = ds - ki * dy[:, :, None]
        dg[:, i] = (ds * old).sum((2, 3))
        ds = ds * carry[:, i, :, None, None]
    group = lambda x: x.unflatten(2, (hk, h // hk)).sum(3)                         # noqa: E731
    return {"dq": group(dq), "dk": group(dk_), "dv": dv_, "dg": dg, "dbeta": dbeta, "dstate": ds}
