"""rls.token_logprobs and rls.distill_loss against their definitions in 64 bits, and their gradients.

Tolerances count roundings of 2^-24 in fp32: a distance d (three, relative), an exponential of it (its exponent's roundings, so 4 |d|), the additions of
a thread and of the joins (n / 256 + 64 in a row), a logarithm; a result in fewer bits is off by half a step of its type more."""
import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def reference(x, tokens, temperature=None, top=0):
    """In 64 bits, on the CPU: logprob, entropy, log p of all entries, the best entries."""
    x = x.cpu().double()
    x = torch.where(x.isnan(), -torch.inf, x).clamp(max=torch.finfo(torch.float32).max)
    rows, n = x.shape
    t = torch.ones(rows, dtype=torch.float64) if temperature is None else temperature.cpu().double()
    t = torch.where(t > 0, t, 1.0)[:, None]
    live = x > -torch.inf
    top_x = x.amax(1, keepdim=True)
    d = torch.where(live, (x - top_x) * (1 / t), -torch.inf)
    log = torch.where(live.any(1, keepdim=True), torch.exp(d).sum(1, keepdim=True).log(), 0.0)
    logp = d - log
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    out = {"logp": logp, "p": p, "entropy": entropy, "log": log[:, 0], "live": live, "inv": 1 / t,
           "d": torch.where(p > 0, d, 0.0).abs().amax(1), "mean_d": torch.where(p > 0, p * d.abs(), 0.0).sum(1)}
    if tokens is not None:
        k = tokens.cpu().long()
        given = (k >= 0) & (k < n)
        out["given"], out["token"] = given, k.clamp(0, n - 1)
        out["logprob"] = torch.where(given, logp.gather(1, out["token"][:, None])[:, 0], 0.0)
    if top:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        best = logp.gather(1, order)
        order = torch.where(live.gather(1, order), order, -1)
        pad = top - order.shape[1]
        out["top_token"] = torch.nn.functional.pad(order, (0, max(0, pad)), value=-1)
        out["top_logprob"] = torch.nn.functional.pad(best, (0, max(0, pad)), value=-torch.inf)
    return out


def steps(n):
    return n / 256 + 64


def near(got, want, tol, what):
    got, want = got.cpu().double(), want.double()
    same = (got == want) | ((got - want).abs() <= tol)
    assert bool(same.all()), (what, float((got - want)[~same].abs().max()), int((~same).sum()))


def check(rls, x, tokens, temperature=None, top=0, workspace=None):
    r = rls.token_logprobs(x, tokens, temperature=temperature, top=top, workspace=workspace)
    w = reference(x, tokens, temperature, top)
    n = x.shape[1]
    by_log = UNIT * (steps(n) + 4 * w["mean_d"] + 4 * w["log"].abs())
    if tokens is not None:
        near(r.logprob, w["logprob"], by_log + UNIT * 4 * w["logprob"].abs(), "logprob")
    near(r.entropy, w["entropy"], (UNIT * (steps(n) + 4 * w["d"])) * (2 + w["mean_d"] + w["log"]), "entropy")
    if top:
        alike = torch.equal(r.top_token.cpu().long(), w["top_token"])
        assert alike, "top_token"
        near(r.top_logprob, w["top_logprob"], (by_log + UNIT * 4 * w["top_logprob"].abs().nan_to_num(posinf=0).amax(1))[:, None], "top")
    near(r.norm[:, 1], w["log"], by_log, "norm")
    return r, w


def logits(rows, n, kind, seed, ld=None, offset=0, spread=3.0):
    gen = torch.Generator().manual_seed(seed)
    whole = (torch.randn(rows * (ld or n) + offset, generator=gen) * spread).to(TYPES[kind]).cuda()
    return whole[offset:].view(rows, ld or n)[:, :n]


def given(rows, n, seed):
    return torch.randint(-1, n + 1, (rows,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


SIZES = [(1, 1), (7, 1), (300, 3), (1, 4), (257, 5), (65, 8), (65, 9), (5, 16), (5, 17), (9, 63), (4, 64), (4, 65), (6, 1000), (3, 1024), (3, 1025), (600, 1027),
         (5, 2049), (3, 8191), (2, 8200), (2, 16385), (1030, 8300), (520, 16500), (3, 40001), (1, 131075), (1, 1 << 20)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n", SIZES)
def test_forward(rls, rows, n, kind):
    x, tokens = logits(rows, n, kind, rows + n), given(rows, n, n)
    temperature = (torch.rand(rows, generator=torch.Generator().manual_seed(n)) + 0.5).cuda()
    for top in (0, 1, 20) if rows * n < 1 << 23 else (0, 20):
        check(rls, x, tokens, temperature if top else None, top)


@pytest.mark.parametrize("n", [1, 3, 16, 40, 300, 1025, 5000, 20000, 70000])
@pytest.mark.parametrize("top", [7, 64, 128])
def test_alternatives_of_equal_and_few_entries(rls, n, top):
    rows = 6
    x = (logits(rows, n, "bf16", n).float() * 0.5).round().to(torch.bfloat16)       # many equal ones
    x[1] = 0.0
    x[1, ::2] = -0.0                                                               # equal ones too
    x[2] = -torch.inf                                                              # nothing left
    x[3] = torch.finfo(torch.bfloat16).min                                         # masked by the lowest value
    x[3, n // 2] = 1.0
    x[4] = torch.nan
    x[4, n - 1] = -3.0
    x[5, n // 3] = torch.inf
    r, _ = check(rls, x, torch.full((rows,), n // 2, dtype=torch.int32, device="cuda"), None, top)
    assert r.logprob[2] == -torch.inf and r.entropy[2] == 0 and r.norm[2].tolist() == [-torch.inf, 0.0] and bool((r.top_token[2] == -1).all())
    assert r.logprob[3] == 0 and r.top_token[4, 0] == n - 1 and r.logprob[5] == (0 if n // 2 == n // 3 else r.logprob[5])


@pytest.mark.parametrize("rows,n", [(1024, 60000), (2, 60000), (600, 20000)])
def test_large_logits_with_few_threads(rls, rows, n):
    """More entries above the threshold than the list holds: packs of 4 that the first 128 of 256 (512, 1024) threads read."""
    x = logits(rows, n, "f32", 1)
    which = torch.arange(n, device="cuda") // 4 % 256 < 128
    x = x + 100.0 * which
    x = x[:2].repeat(rows // 2, 1) if rows > 600 else x
    got = rls.token_logprobs(x.contiguous(), None, top=128)
    want = torch.sort(x[:2], dim=1, descending=True, stable=True).indices[:, :128]
    assert torch.equal(got.top_token[:2].long(), want)
    sorted_up = torch.arange(n, dtype=torch.float32, device="cuda").expand(2, n).contiguous()
    for y in (sorted_up, -sorted_up):
        assert torch.equal(rls.token_logprobs(y, None, top=100).top_token.long(), torch.sort(y, dim=1, descending=True, stable=True).indices[:, :100])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n,ld,offset", [(5, 3, 7, 1), (4, 30, 31, 3), (6, 1001, 1003, 1), (3, 4000, 4001, 5), (2, 20001, 20011, 7)])
def test_strides(rls, kind, rows, n, ld, offset):
    x, tokens = logits(rows, n, kind, n, ld, offset), given(rows, n, n)
    r, w = check(rls, x, tokens, None, min(n, 9))
    gradient(rls, x, tokens, r, w, seed=n)
    same = rls.token_logprobs(x.contiguous(), tokens, top=min(n, 9))
    assert torch.equal(r.logprob, same.logprob) and torch.equal(r.top_token, same.top_token)


def gradient(rls, x, tokens, r, w, temperature=None, seed=0, out=None, which="both"):
    gen = torch.Generator().manual_seed(seed)
    rows, n = x.shape
    dlp, dh = torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()
    dlp, dh = (dlp if which != "entropy" else None), (dh if which != "logprob" else None)
    before = x.clone()
    got = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, dlp, dh, temperature=temperature, out=out)
    a = torch.zeros(rows, 1, dtype=torch.float64) if dlp is None else (dlp.cpu().double() * w["given"])[:, None]
    c = torch.zeros(rows, 1, dtype=torch.float64) if dh is None else dh.cpu().double()[:, None]
    lp = torch.where(w["p"] > 0, w["logp"], 0.0)
    want = -w["p"] * (a + c * (lp + w["entropy"][:, None]))
    want.scatter_add_(1, w["token"][:, None], a)
    want = torch.where(w["live"], want * w["inv"], 0.0)
    size = w["p"] * (a.abs() + c.abs() * (lp.abs() + w["entropy"][:, None]))
    size.scatter_add_(1, w["token"][:, None], a.abs())
    # an exponential whose exponent is off by roundings of d and L, then four operations
    off = UNIT * (8 + steps(n) + 4 * (lp.abs() + 2 * w["log"][:, None] + w["mean_d"][:, None]))
    off = off + (UNIT * (steps(n) + 4 * w["d"]) * (2 + w["mean_d"] + w["log"]))[:, None]      # the entropy's own
    kind = torch.finfo(before.dtype)
    near(got, want, size * w["inv"] * off + want.abs() * kind.eps / 2 * (1 + 1e-6) + kind.smallest_normal * kind.eps + 1e-37, "dlogits")
    return got


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n", [s for s in SIZES if s[0] * s[1] < 1 << 23])
def test_backward(rls, rows, n, kind):
    x, tokens = logits(rows, n, kind, rows + n), given(rows, n, n)
    temperature = (torch.rand(rows, generator=torch.Generator().manual_seed(n)) + 0.5).cuda()
    for t, which in ((None, "both"), (temperature, "both"), (None, "logprob"), (temperature, "entropy")):
        r, w = check(rls, x, tokens, t)
        gradient(rls, x, tokens, r, w, t, n, which=which)


@pytest.mark.parametrize("n", [2, 5, 16, 50, 1500, 30000])
def test_masks_in_the_gradient(rls, n):
    x = logits(6, n, "f32", n)
    x[0, n // 2] = -torch.inf                                                      # the given token is masked
    x[1] = -torch.inf
    x[2, : n // 2] = torch.nan
    x[3, 0] = torch.finfo(torch.float32).min
    x[4] = torch.finfo(torch.float32).min
    x[5] *= 1e4
    tokens = torch.full((6,), n // 2, dtype=torch.int32, device="cuda")
    r, w = check(rls, x, tokens, None, 2)
    got = gradient(rls, x, tokens, r, w, None, n)
    assert bool(got.isfinite().all()) and not got[1].any() and not got[2, : n // 2].any() and got[0, n // 2] == 0


def test_temperatures(rls):
    x, tokens = logits(8, 100, "f32", 0), given(8, 100, 0)
    t = torch.tensor([0.0, -1.0, torch.nan, torch.inf, 1e-3, 1e-40, 1e30, 3e38]).cuda()
    x[:, 5] = -torch.inf
    r = rls.token_logprobs(x, tokens, temperature=t, top=3)
    plain = rls.token_logprobs(x, tokens, top=3)
    assert torch.equal(r.logprob[:3], plain.logprob[:3]) and torch.equal(r.entropy[:3], plain.entropy[:3]) and torch.equal(r.top_token, plain.top_token)
    flat = torch.log(torch.tensor(99.0))
    for i in (3, 6, 7):
        assert abs(float(r.entropy[i]) - flat) < 1e-5 and torch.allclose(r.top_logprob[i].cpu(), -flat.expand(3), atol=1e-5)
    assert r.top_logprob[5, 0] == 0 and r.entropy[5] == 0
    g = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, torch.ones(8, device="cuda"), torch.ones(8, device="cuda"), temperature=t)
    assert not g.isnan().any() and not g[:, 5].any()


def test_agrees_with_sample(rls):
    """The log-probability of a draw is the one that the draw itself reports."""
    for rows, n in ((1000, 3), (50, 777), (4, 40000)):
        x = logits(rows, n, "bf16", n)
        t = (torch.rand(rows, generator=torch.Generator().manual_seed(n)) + 0.5).cuda()
        token, logprob = rls.sample(x, torch.rand(rows, generator=torch.Generator().manual_seed(n)).cuda(), temperature=t)
        near(rls.token_logprobs(x, token, temperature=t).logprob, logprob.cpu(), UNIT * (2 * steps(n) + 200) + n * 2.0 ** -39, "sample")


@pytest.mark.parametrize("n", [3, 60, 3000])
def test_autograd(rls, n):
    x = logits(40, n, "f32", n).clone().requires_grad_()
    tokens = given(40, n, n).clamp(0, n - 1)
    by = torch.randn(40, generator=torch.Generator().manual_seed(1)).cuda()
    for what in ("both", "logprob", "entropy"):
        r = rls.token_logprobs(x, tokens, top=2)
        logp = torch.log_softmax(x.double(), 1)
        parts = {"logprob": ((r.logprob * by).sum(), (logp.gather(1, tokens.long()[:, None])[:, 0] * by).sum()),
                 "entropy": (r.entropy.sum(), -(logp.exp() * logp).sum())}
        mine, plain = (sum(v[i] for k, v in parts.items() if what in (k, "both")) for i in (0, 1))
        assert not r.norm.requires_grad and not r.top_logprob.requires_grad
        near(torch.autograd.grad(mine, x)[0], torch.autograd.grad(plain, x)[0].cpu(), UNIT * (steps(n) + 400) * 8, what)
    # against differences: the slope along a direction (step 2^-7: a third-order term of at most step^2 times the sum of the factors, roundings over the step)
    way = torch.randn(40, n, generator=torch.Generator().manual_seed(2)).cuda()
    value = lambda y: (lambda r: (r.logprob * by).double().sum() + r.entropy.double().sum())(rls.token_logprobs(y, tokens))       # noqa: E731
    with torch.no_grad():
        h = 2.0 ** -7
        slope = (value(x + h * way) - value(x - h * way)) / (2 * h)
    r = rls.token_logprobs(x, tokens)
    got = (torch.autograd.grad((r.logprob * by).sum() + r.entropy.sum(), x)[0] * way).double().sum()
    assert abs(float(slope - got)) < 40 * (h * h * 64 + UNIT * (steps(n) + 200) * 20 / h)


# ---- distillation ----------------------------------------------------------------------------------------------------

def taught(rows, n, k, kind, seed):
    gen = torch.Generator().manual_seed(seed)
    tokens = torch.randint(-1, n + 1, (rows, k), generator=gen, dtype=torch.int32)
    scores = (torch.randn(rows, k, generator=gen) * 2).to(TYPES[kind])
    if rows > 3:
        scores[1] = -torch.inf                                                     # no entry
        tokens[2] = -1
        tokens[3] = min(n - 1, 2)                                                  # the same one every time
        scores[0, 0] = torch.nan
    return tokens.cuda(), scores.cuda()


def taught_reference(x, tokens, scores, temperature):
    w = reference(x, None, temperature)
    n = x.shape[1]
    k, s = tokens.cpu().long(), scores.cpu().double()
    s = torch.where((k >= 0) & (k < n) & ~s.isnan(), s, -torch.inf)
    s = s * w["inv"]
    some = (s > -torch.inf).any(1, keepdim=True)
    p = torch.where(some, torch.softmax(torch.where(some, s, 0.0), 1), 0.0)
    logp = torch.where(p > 0, s - torch.logsumexp(torch.where(some, s, 0.0), 1, keepdim=True), 0.0)
    logq = w["logp"].gather(1, k.clamp(0, n - 1))
    w["loss"] = torch.where(p > 0, p * (logp - logq), 0.0).sum(1)
    w["size"] = torch.where(p > 0, p * (logp.abs() + logq.abs().nan_to_num(posinf=0)), 0.0).sum(1)
    w["target"] = torch.zeros_like(w["p"]).scatter_add_(1, k.clamp(0, n - 1), p)
    w["some"] = some
    w["spread"] = torch.where(p > 0, s - s.amax(1, keepdim=True), 0.0).abs().amax(1)
    return w


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (6, 3, 5), (70, 16, 4), (9, 17, 128), (5, 64, 64), (5, 700, 65), (6, 1025, 8), (1030, 2100, 3), (5, 9000, 32), (4, 20001, 100),
                                      (1, 140001, 128)])
def test_distill(rls, rows, n, k, kind):
    x = logits(rows, n, kind, n)
    temperature = (torch.rand(rows, generator=torch.Generator().manual_seed(n)) + 0.5).cuda()
    dloss = torch.randn(rows, generator=torch.Generator().manual_seed(k)).cuda()
    for teacher in TYPES:
        tokens, scores = taught(rows, n, k, teacher, n + k)
        for t in (None, temperature):
            loss, norm = rls.distill_loss(x, tokens, scores, temperature=t)
            w = taught_reference(x, tokens, scores, t)
            by_log = UNIT * (steps(n) + 4 * w["mean_d"] + 4 * w["log"].abs())
            # p: roundings of an exponential, of a sum over 128 and of a division, times what it weighs
            near(loss, w["loss"], by_log + UNIT * (4 * w["spread"] + 32) * w["size"], "loss")
            got = rls.distill_loss_backward(x, tokens, scores, norm, dloss, temperature=t)
            g = dloss.cpu().double()[:, None] * w["inv"] * w["some"]
            want = g * (w["p"] - w["target"])
            lp = torch.where(w["p"] > 0, w["logp"], 0.0).abs()
            off = w["p"] * (UNIT * (8 + 4 * lp) + 2 * by_log[:, None]) + w["target"] * (UNIT * (32 + k + 4 * w["spread"]))[:, None]
            f = torch.finfo(x.dtype)
            near(got, want, g.abs() * off + want.abs() * (f.eps / 2) * (1 + 1e-6) + 4 * UNIT * want.abs() + f.smallest_normal * f.eps + 1e-37, "dlogits")


def test_distill_masks(rls):
    for n in (20, 5000, 30000):
        x = logits(4, n, "f32", n)
        x[0, 3] = -torch.inf
        x[1] = -torch.inf
        x[2, :5] = torch.nan
        tokens = torch.tensor([[3, 4], [3, 4], [7, 8], [7, 8]], dtype=torch.int32, device="cuda")
        scores = torch.tensor([[0.0, 1.0], [0.0, 1.0], [0.0, 1.0], [0.0, -1e30]], device="cuda")
        loss, norm = rls.distill_loss(x, tokens, scores)
        assert loss[0] == torch.inf and loss[1] == torch.inf and bool(loss[2:].isfinite().all())
        g = rls.distill_loss_backward(x, tokens, scores, norm, torch.ones(4, device="cuda"))
        assert bool(g.isfinite().all()) and g[0, 3] == 0 and not g[1].any() and not g[2, :5].any()
        assert abs(float(g[3, 7]) + 1 - float(torch.softmax(x[3], 0)[7])) < 1e-6      # the entry without weight adds nothing
        # a masked entry without weight costs nothing
        assert rls.distill_loss(x[:1], tokens[:1], torch.tensor([[-torch.inf, 0.0]], device="cuda"))[0].isfinite().all()


def test_teacher_is_what_alternatives_list(rls):
    """A student that is its own teacher: the loss is the logarithm of the mass beyond the list, taken off; with the whole row listed, 0."""
    x = logits(5, 100, "f32", 3)
    r = rls.token_logprobs(x, None, top=100)
    loss, _ = rls.distill_loss(x, r.top_token, r.top_logprob)
    near(loss, torch.zeros(5), UNIT * 400, "whole row")
    r = rls.token_logprobs(x, None, top=10)
    loss, _ = rls.distill_loss(x, r.top_token, r.top_logprob)
    near(loss, -r.top_logprob.double().exp().sum(1).log().cpu(), UNIT * 800, "ten")


def test_distill_autograd(rls):
    x = logits(30, 500, "f32", 3).clone().requires_grad_()
    tokens, scores = taught(30, 500, 6, "f32", 4)
    weight = torch.rand(30, generator=torch.Generator().manual_seed(1)).cuda()
    loss, norm = rls.distill_loss(x, tokens, scores)
    assert not norm.requires_grad
    got = torch.autograd.grad((loss * weight).sum(), x)[0]
    w = taught_reference(x.detach(), tokens, scores, None)
    near(got, weight.cpu().double()[:, None] * w["some"] * (w["p"] - w["target"]), UNIT * 1000, "dlogits")


# ---- how they are called -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n", [(300, 3), (50, 700), (6, 30001)])
def test_gradients_in_place(rls, kind, rows, n):
    x, tokens = logits(rows, n, kind, 1), given(rows, n, 2)
    r = rls.token_logprobs(x, tokens)
    by = torch.randn(rows, generator=torch.Generator().manual_seed(3)).cuda()
    want = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, by, by)
    same = x.clone()
    assert rls.token_logprobs_backward(same, tokens, r.norm, r.entropy, by, by, out=same) is same and torch.equal(same, want)
    k, s = taught(rows, n, 20, "f32", 5)
    _, norm = rls.distill_loss(x, k, s)
    want = rls.distill_loss_backward(x, k, s, norm, by)
    same, version = x.clone(), x._version
    rls.distill_loss_backward(same, k, s, norm, by, out=same)
    assert torch.equal(same, want) and same._version > version
    wide = torch.full((rows, n + 3), 7.0, dtype=x.dtype, device="cuda")               # rows further apart: what lies between stays
    rls.distill_loss_backward(x, k, s, norm, by, out=wide[:, :n])
    assert torch.equal(wide[:, :n], want) and bool((wide[:, n:] == 7).all())


def test_graph_and_streams(rls):
    """Captured calls replayed with new inputs between eager ones, and calls on several streams at once, each with its own workspace."""
    rows, n = 4, 50001
    x, tokens = logits(rows, n, "bf16", 1), given(rows, n, 1)
    k, s = taught(rows, n, 16, "f32", 2)
    ws = [torch.empty(rls.token_logprobs_workspace_bytes(rows, n, 20) + 256, dtype=torch.uint8, device="cuda") for _ in range(2)]
    by = torch.randn(rows, generator=torch.Generator().manual_seed(3)).cuda()

    def all_of(x, spaces):
        r = rls.token_logprobs(x, tokens, top=20, workspace=spaces[0])
        d = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, by, by)
        loss, norm = rls.distill_loss(x, k, s, workspace=spaces[1])
        return (*r, d, loss, norm, rls.distill_loss_backward(x, k, s, norm, by))
    all_of(x, ws)
    torch.cuda.synchronize()
    held = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of(held, ws)
    for seed in range(4):
        held.copy_(logits(rows, n, "bf16", 10 + seed))
        want = all_of(held, [None, None])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
    streams = [torch.cuda.Stream() for _ in range(3)]
    xs = [logits(rows, n, "bf16", 20 + i) for i in range(3)]
    want = [all_of(x, [None, None]) for x in xs]
    torch.cuda.synchronize()
    got = []
    for st, x in zip(streams, xs):
        with torch.cuda.stream(st):
            got.append([all_of(x, [None, None]) for _ in range(3)][-1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_past_32_bits(rls):
    """Rows that begin beyond 2^31 entries: the last ones, against the same rows by themselves."""
    rows, n = 33, 1 << 26 >> 2
    x = torch.empty((rows + 100) * n, dtype=torch.bfloat16, device="cuda").view(rows + 100, n)
    x[-2:] = logits(2, n, "bf16", 1)
    x[:-2] = 0
    tokens = torch.full((rows + 100,), n - 1, dtype=torch.int32, device="cuda")
    r, few = rls.token_logprobs(x, tokens, top=4), rls.token_logprobs(x[-2:].clone(), tokens[-2:].clone(), top=4)
    assert torch.equal(r.top_token[-2:], few.top_token)
    near(r.logprob[-2:], few.logprob.cpu(), UNIT * 2 * steps(n), "logprob")
    g = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, torch.ones(rows + 100, device="cuda"), out=x)
    w = few.norm.clone()
    assert float(g[-1, n - 1]) > 0.9 and g[0, 0] < 0 and bool(w.isfinite().all())


@pytest.mark.parametrize("n", [3, 18])
def test_many_rows(rls, n):
    """More rows than a launch takes: the first and the last ones against the same rows by themselves."""
    rows = (1 << 21) + 9
    x = torch.randn(rows, n, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda")
    tokens = torch.arange(rows, dtype=torch.int32, device="cuda") % n
    r = rls.token_logprobs(x, tokens, top=2)
    by = torch.ones(rows, device="cuda")
    g = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, by, by)
    k, s = tokens[:, None].contiguous(), by[:, None].contiguous()
    loss, norm = rls.distill_loss(x, k, s)
    d = rls.distill_loss_backward(x, k, s, norm, by)
    for part in (slice(0, 50), slice((1 << 21) - 20, rows)):
        px, pt = x[part].clone(), tokens[part].clone()
        q = rls.token_logprobs(px, pt, top=2)
        assert all(torch.equal(a[part], b) for a, b in zip(r, q))
        assert torch.equal(g[part], rls.token_logprobs_backward(px, pt, q.norm, q.entropy, by[part].clone(), by[part].clone()))
        pl, pn = rls.distill_loss(px, k[part].clone(), s[part].clone())
        assert torch.equal(loss[part], pl) and torch.equal(d[part], rls.distill_loss_backward(px, k[part].clone(), s[part].clone(), pn, by[part].clone()))
