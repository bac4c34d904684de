"""Performance cases of the training step's operators around the gradient codec.

What a data-parallel training program does on one GPU before its gradients are
encoded and after they are decoded: the embedding lookup and its gradient for
every simulated rank (the rank gradients that the codec takes), the global
norm of the decoded gradients with the clip coefficient, and the AdamW step
over all of a model's tensors, with its moments in float32 or in FP8 E4M3
codes with one scale per 256 elements.

Sizes are those of the repository's own workloads (hidden 256; hidden 1024
with MLP 2816; hidden 1536 with MLP 4096; 32000 tokens), odd ones beside them;
:func:`draw` spreads over the ranges between and around them.  Gradients are
Student-t(3) noise of rms 2.15e-4, tokens follow Zipf's law, moments are those
of a run under way.

A model's tensors live in one flat buffer each for parameters, gradients and
moments, every tensor starting at a multiple of 512 elements; what lies
between two tensors is zero and stays so.
"""

import math

import torch

own = False

RMS = 2.15e-4
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.95, 1e-8, 0.1
MAX_NORM = 1.0
SEED = 20
ALIGN = 512         # elements between the starts of two tensors
BLOCK = 256         # elements under one scale of an 8-bit moment
MASK = 0xFFFFFFFF


def listed():
    return [
        # one generated token for each of 16 sequences: launch and latency
        dict(name="lookup_generate", kind="lookup", T=16, V=32000, d=1024, table="bf16", out="bf16", ids=64, pads=False),
        # a training batch of the 600M model, from the float32 master table
        dict(name="lookup_batch_600m", kind="lookup", T=65536, V=32000, d=1536, table="f32", out="bf16", ids=32,
             pads=False),
        # one short sequence of a small model: launches count
        dict(name="embgrad_small", kind="embgrad", N=1, T=512, V=4096, d=256, grad="f32", ids=64, pads=False,
             accumulate=False),
        # the eight ranks' embedding gradients of the 300M model, as the codec takes them
        dict(name="embgrad_ranks_300m", kind="embgrad", N=8, T=2048, V=32000, d=1024, grad="bf16", ids=64, pads=False,
             accumulate=False),
        # a tied table: the lookup's share is added to the gradient that the output layer left there
        dict(name="embgrad_tied_600m", kind="embgrad", N=1, T=65536, V=32000, d=1536, grad="bf16", ids=32, pads=False,
             accumulate=True),
        # a width and a vocabulary that nothing divides, padded sequences
        dict(name="embgrad_odd", kind="embgrad", N=3, T=5001, V=50001, d=771, grad="bf16", ids=64, pads=True,
             accumulate=False),
        # the norm of a small model's gradients: latency
        dict(name="norm_small", kind="norm", layers=1, hidden=256, mlp=704, vocab=0, grad="f32"),
        # the norm over every decoded gradient of the 300M model
        dict(name="norm_300m", kind="norm", layers=24, hidden=1024, mlp=2816, vocab=32000, grad="f32"),
        # one small layer's step: latency
        dict(name="adamw_small", kind="adamw", layers=1, hidden=256, mlp=704, vocab=0, grad="f32", state="f32",
             copy=False),
        # the whole 300M model, with the bfloat16 weights that the next forward pass reads
        dict(name="adamw_300m", kind="adamw", layers=24, hidden=1024, mlp=2816, vocab=32000, grad="f32", state="f32",
             copy=True),
        # tensors that no vector width divides, 8-bit moments
        dict(name="adamw8_odd", kind="adamw", layers=3, hidden=515, mlp=1373, vocab=0, grad="bf16", state="e4m3",
             copy=True),
        # the whole 600M model with 8-bit moments
        dict(name="adamw8_600m", kind="adamw", layers=24, hidden=1536, mlp=4096, vocab=0, grad="f32", state="e4m3",
             copy=True),
    ]


def _spread(rng, lo, hi, odd=0.3, step=8):
    """A size between lo and hi, spread over its logarithm; a multiple of `step` but for a share of odd ones."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < odd:
        return v
    return max(lo, v // step * step)


def draw(rng):
    kind = rng.choice(["lookup", "embgrad", "embgrad", "norm", "adamw", "adamw"])
    if kind == "lookup":
        return dict(kind=kind, T=_spread(rng, 1, 65536, 0.5), V=_spread(rng, 1000, 131072), d=_spread(rng, 64, 1536),
                    table=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16", "bf16"]), ids=rng.choice([32, 64]),
                    pads=rng.random() < 0.3)
    if kind == "embgrad":
        N = rng.choice([1, 1, 2, 4, 8, rng.randint(3, 16)])
        T, V, d = _spread(rng, 1, 65536 // N, 0.5), _spread(rng, 1000, 131072), _spread(rng, 64, 1536)
        while N * V * d > 8 * 32000 * 1024:
            V = V // 2 + 1
        return dict(kind=kind, N=N, T=T, V=V, d=d, grad=rng.choice(["f32", "bf16", "bf16"]), ids=rng.choice([32, 64]),
                    pads=rng.random() < 0.3, accumulate=rng.random() < 0.3)
    hidden = _spread(rng, 64, 1536)
    case = dict(kind=kind, layers=rng.randint(1, 24), hidden=hidden, mlp=hidden * 8 // 3 + rng.randint(0, 7),
                vocab=rng.choice([0, 0, _spread(rng, 1000, 32000)]), grad=rng.choice(["f32", "f32", "bf16"]))
    if kind == "adamw":
        case.update(state=rng.choice(["f32", "e4m3"]), copy=rng.random() < 0.5)
    while case["layers"] > 1 and work(case)["bytes"] > 1e10:
        case["layers"] -= 1
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _noise(gen, shape, dev):
    """Student-t(3) noise of rms about 2.15e-4."""
    chi2 = torch.zeros(shape, device=dev)
    for _ in range(3):
        chi2 += torch.randn(shape, generator=gen, device=dev).square_()
    return torch.randn(shape, generator=gen, device=dev).div_(chi2.sqrt_()).mul_(RMS)


def _tokens(gen, shape, V, bits, pads, dev):
    """Ids by Zipf's law; with `pads` the last eighth of every sequence is -1."""
    u = torch.rand(shape, generator=gen, device=dev, dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    if pads:
        ids[..., shape[-1] - shape[-1] // 8:] = -1
    return ids.to(torch.int64 if bits == 64 else torch.int32)


def _shapes(case):
    """Shapes of a model's tensors: those with weight decay (matrices), then those without (norm vectors)."""
    h, f, L = case["hidden"], case["mlp"], case["layers"]
    mats = [(h, h)] * 4 + [(f, h)] * 2 + [(h, f)]
    table = [(case["vocab"], h)] * 2 if case["vocab"] else []
    return mats * L + table, [(h,)] * (2 * L + 1)


class Layout:
    """Where each of a model's tensors lies in the flat buffers."""

    def __init__(self, case):
        decayed, plain = _shapes(case)
        self.shapes = decayed + plain
        self.decay = [DECAY] * len(decayed) + [0.0] * len(plain)
        self.starts, at = [], 0
        for s in self.shapes:
            self.starts.append(at)
            at += (math.prod(s) + ALIGN - 1) // ALIGN * ALIGN
        self.total = at
        self.split = self.starts[len(decayed)]
        self.elements = sum(math.prod(s) for s in self.shapes)

    def views(self, flat):
        return [flat[a:a + math.prod(s)].view(s) for a, s in zip(self.starts, self.shapes)]

    def inside(self, dev):
        """True where a position of the flat buffers belongs to a tensor."""
        ends = torch.tensor([a + math.prod(s) for a, s in zip(self.starts, self.shapes)], device=dev)
        starts = torch.tensor(self.starts, device=dev)
        at = torch.arange(self.total, device=dev)
        return at < ends[torch.searchsorted(starts, at, right=True) - 1]

    def calls(self, dev):
        """Tensor index and number within its tensor of every group of 512 elements."""
        counts = torch.tensor([(math.prod(s) + ALIGN - 1) // ALIGN for s in self.shapes], device=dev)
        tensor = torch.repeat_interleave(torch.arange(len(self.shapes), device=dev), counts)
        first = torch.cumsum(counts, 0) - counts
        return tensor, torch.arange(self.total // ALIGN, device=dev) - first[tensor]


def _gradients(case, lay, gen, dev):
    g = _noise(gen, lay.total, dev)
    g *= lay.inside(dev)
    return g.to(DTYPES[case["grad"]])


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    kind = case["kind"]
    if kind == "lookup":
        T, V, d = case["T"], case["V"], case["d"]
        return dict(case=case, tokens=_tokens(gen, (T,), V, case["ids"], case["pads"], dev),
                    table=(torch.randn((V, d), generator=gen, device=dev) * 0.02).to(DTYPES[case["table"]]),
                    out=torch.empty((T, d), dtype=DTYPES[case["out"]], device=dev))
    if kind == "embgrad":
        N, T, V, d = (case[k] for k in "NTVd")
        grads = _noise(gen, (N, V, d), dev) if case["accumulate"] else torch.zeros((N, V, d), device=dev)
        return dict(case=case, tokens=_tokens(gen, (N, T), V, case["ids"], case["pads"], dev),
                    dout=_noise(gen, (N, T, d), dev).to(DTYPES[case["grad"]]), grads=grads)
    lay = Layout(case)
    grads = _gradients(case, lay, gen, dev)
    if kind == "norm":
        return dict(case=case, grads=lay.views(grads), flat=grads, out=torch.empty(2, device=dev))
    inside = lay.inside(dev)
    params = torch.randn(lay.total, generator=gen, device=dev).mul_(0.02).mul_(inside)
    m = _noise(gen, lay.total, dev).mul_(0.3).mul_(inside)
    v = torch.randn(lay.total, generator=gen, device=dev).exp_().mul_(RMS * RMS).mul_(inside)
    state = dict(case=case, layout=lay, calls=lay.calls(dev), params=params, grads=grads, step=100,
                 clip=torch.full((1,), 0.7, device=dev),
                 copy=params.to(torch.bfloat16) if case["copy"] else None)
    if case["state"] == "f32":
        return dict(state, m=m, v=v)
    for name, x in (("m", m), ("v", v)):
        x = x.view(-1, BLOCK)
        scale = x.abs().amax(1) / 448
        codes = (x / scale.clamp(min=1e-38)[:, None]).clamp_(-448, 448)
        state[name] = codes.to(torch.float8_e4m3fn).view(torch.uint8).view(-1)
        state[name + "_scales"] = scale
    return state


# ---------------------------------------------------------------------------
# The operators' plain forms
# ---------------------------------------------------------------------------

def _scale(case):
    return math.sqrt(case["d"])


def _plain_lookup(s):
    table, tokens = s["table"], s["tokens"].long()
    V = table.shape[0]
    valid = (tokens >= 0) & (tokens < V)
    rows = table[tokens.clamp(0, V - 1)].float() * _scale(s["case"])
    return torch.where(valid[:, None], rows, 0.0).to(s["out"].dtype)


def _plain_embgrad(s):
    case, grads = s["case"], s["grads"]
    N, T, V, d = (case[k] for k in "NTVd")
    tokens = s["tokens"].long()
    valid = (tokens >= 0) & (tokens < V)
    rows = (tokens.clamp(0, V - 1) + torch.arange(N, device=tokens.device)[:, None] * V).view(-1)
    dout = torch.where(valid[..., None], s["dout"].float(), 0.0).view(-1, d)
    sums = torch.zeros((N * V, d), device=grads.device).index_add_(0, rows, dout) * _scale(case)
    if case["accumulate"]:
        grads.view(-1, d).add_(sums)
    else:
        grads.view(-1, d).copy_(sums)
    return grads


def _plain_norm(s):
    norm = s["flat"].double().square().sum().sqrt()
    coef = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    return torch.stack([norm, torch.where(torch.isfinite(norm), coef, math.nan)]).float()


def _random_words(calls, step, lanes):
    """The four words of Philox4x32-10 for every 8 elements, as whole numbers of 64 bits: [groups of 512, 64, 4]."""
    tensor, number = calls
    c0 = number[:, None] * 64 + lanes
    c = [c0 & MASK, c0 >> 32, tensor[:, None].expand_as(c0), torch.full_like(c0, step & MASK)]
    k0, k1 = SEED & MASK, SEED >> 32
    for r in range(10):
        if r:
            k0, k1 = (k0 + 0x9E3779B9) & MASK, (k1 + 0xBB67AE85) & MASK
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((p1 >> 32) & MASK) ^ c[1] ^ k0, p1 & MASK, ((p0 >> 32) & MASK) ^ c[3] ^ k1, p0 & MASK]
    return torch.stack(c, -1)


def _random_numbers(s):
    """One number of 16 bits for every element: [blocks, 256]."""
    lanes = torch.arange(64, device=s["params"].device)
    w = _random_words(s["calls"], s["step"], lanes)
    halves = torch.stack([w & 0xFFFF, w >> 16], -1)                         # [groups, lane, word, half]
    return halves.view(-1, 64, 2, 4).transpose(1, 2).reshape(-1, BLOCK)     # words 0, 1: first block; 2, 3: second


def _plain_codes(x, r, keep):
    """E4M3 values and scales of blocks x [blocks, 256], rounded by the numbers r; `keep`: nothing positive becomes 0."""
    amax = x.abs().amax(1)
    mult = torch.where(amax == 0, 0.0, 448 / amax).clamp(max=torch.finfo(torch.float32).max)
    y = x * mult[:, None]
    a = y.abs()
    low = a < 2.0 ** -6
    t = torch.where(low, a + 2.0 ** -6, a)
    q = ((t.view(torch.int32) + (r.int() * 16 + 8)) & -0x100000).view(torch.float32)
    q = torch.where(low, q - 2.0 ** -6, q).clamp(max=448.0)
    if keep:
        q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q)
    return torch.copysign(q, y), amax / 448


def _plain_adamw(s):
    case, lay, p = s["case"], s["layout"], s["params"]
    eight = case["state"] == "e4m3"
    s["step"] += 1
    c1, c2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    g = s["grads"].float() * s["clip"]
    m, v = s["m"], s["v"]
    if eight:
        m = (m.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["m_scales"][:, None]).view(-1)
        v = (v.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["v_scales"][:, None]).view(-1)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    update = m / (v.sqrt() * (1 / math.sqrt(c2)) + EPS)
    p[:lay.split] *= 1 - LR * DECAY
    p -= update * (LR / c1)
    if eight:
        r = _random_numbers(s)
        for name, x in (("m", m), ("v", v)):
            q, scale = _plain_codes(x.view(-1, BLOCK), r, name == "v")
            s[name] = q.to(torch.float8_e4m3fn).view(torch.uint8).view(-1)
            s[name + "_scales"] = scale
    else:
        s["m"], s["v"] = m, v
    if s["copy"] is not None:
        s["copy"].copy_(p)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

_contexts = {}


def _context(s):
    """The program's context on the stream of the state's first pass."""
    if "context" not in s:
        import paper_2607_07494_amd as gift
        stream = torch.cuda.current_stream()
        key = (stream.device_index, stream.cuda_stream)
        if key not in _contexts:
            _contexts[key] = gift.Context()
        s["context"] = _contexts[key]
    return s["context"]


def _own_pass(s):
    import paper_2607_07494_amd as gift
    ctx, case, kind = _context(s), s["case"], s["case"]["kind"]
    if kind == "lookup":
        gift.embedding(ctx, s["table"], s["tokens"], s["out"], scale=_scale(case))
        return s["out"]
    if kind == "embgrad":
        gift.embedding_grad(ctx, s["tokens"], s["dout"], s["grads"], scale=_scale(case), accumulate=case["accumulate"])
        return s["grads"]
    if kind == "norm":
        gift.grad_norm(ctx, s["grads"], s["out"], max_norm=MAX_NORM)
        return s["out"]
    if "optimizer" not in s:    # the program's optimizer, on its parameters and moments
        lay = s["layout"]
        names = ("m", "v") if case["state"] == "f32" else ("m", "v", "m_scales", "v_scales")
        s["optimizer"] = gift.AdamW(
            ctx, lay.views(s["params"]), betas=(BETA1, BETA2), eps=EPS, weight_decay=lay.decay, moments=case["state"],
            seed=SEED, state={k: s[k] for k in names}, copies=lay.views(s["copy"]) if case["copy"] else None)
        s["grad_views"] = lay.views(s["grads"])
    s["step"] += 1
    s["optimizer"].step(s["grad_views"], lr=LR, step=s["step"], grad_scale=s["clip"])


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        result = _own_pass(s)
    else:
        result = {"lookup": _plain_lookup, "embgrad": _plain_embgrad, "norm": _plain_norm, "adamw": _plain_adamw}[kind](s)
    if kind != "adamw":
        return result
    out = {"params": s["params"], "m": s["m"], "v": s["v"]}
    if s["case"]["state"] == "e4m3":
        out = {"params": s["params"], "m": s["m"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn),
               "m_scales": s["m_scales"], "v_scales": s["v_scales"]}
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


# ---------------------------------------------------------------------------
# Minimal work
# ---------------------------------------------------------------------------

def _distinct(T, V):
    """Distinct ids expected among T drawn by :func:`_tokens`' law from V."""
    p = torch.log1p(1 / torch.arange(1, V + 1, dtype=torch.float64)) / math.log(V + 1.0)
    return float(-torch.expm1(T * torch.log1p(-p)).sum())


def work(case):
    kind = case["kind"]
    if kind == "lookup":
        T, d = case["T"], case["d"]
        valid = T - (T // 8 if case["pads"] else 0)
        rows = _distinct(valid, case["V"])
        return {"bytes": T * case["ids"] // 8 + rows * d * BYTES[case["table"]] + T * d * BYTES[case["out"]],
                "flops": valid * d}
    if kind == "embgrad":
        N, T, V, d = (case[k] for k in "NTVd")
        valid = T - (T // 8 if case["pads"] else 0)
        rows = _distinct(valid, V)
        written = 2 * rows * d * 4 if case["accumulate"] else V * d * 4
        return {"bytes": N * (T * case["ids"] // 8 + valid * d * BYTES[case["grad"]] + written),
                "flops": N * (valid + rows) * d}
    n = Layout(case).elements
    if kind == "norm":
        return {"bytes": n * BYTES[case["grad"]] + 8, "flops": 2 * n}
    moments = 16 if case["state"] == "f32" else 4 + 16 / BLOCK
    return {"bytes": n * (8 + BYTES[case["grad"]] + moments + (2 if case["copy"] else 0)), "flops": 16 * n}


# ---------------------------------------------------------------------------
# Results in 64 bits
# ---------------------------------------------------------------------------

def _exact_codes(x, r, keep):
    """Block rounding of float64 blocks: the two neighbours on E4M3's grid, the upper one where the number says so."""
    amax = x.abs().amax(1)
    y = torch.where(amax[:, None] > 0, x * 448 / amax.clamp(min=1e-300)[:, None], 0.0)
    a = y.abs()
    grid = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    grid = torch.where(a / grid >= 16, grid * 2, grid)      # where the logarithm's rounding took the lower octave
    grid = torch.where((a / grid < 8) & (grid > 2.0 ** -9), grid / 2, grid)
    low = torch.floor(a / grid)
    up = a / grid - low + (r + 0.5) / 65536 >= 1
    q = ((low + up) * grid).clamp(max=448.0)
    if keep:
        q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q)
    return torch.copysign(q, y), amax / 448


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "lookup":
        V = case["V"]
        table = torch.cat([s["table"].double() * _scale(case), torch.zeros((1, case["d"]), device=_device()).double()])
        tokens = s["tokens"].long()
        return table[torch.where((tokens < 0) | (tokens >= V), V, tokens)]
    if kind == "embgrad":
        V = case["V"]
        out = s["grads"].double()
        for j in range(case["N"]):
            keep = (s["tokens"][j] >= 0) & (s["tokens"][j] < V)
            out[j].index_add_(0, s["tokens"][j][keep].long(), s["dout"][j][keep].double(), alpha=_scale(case))
        return out
    if kind == "norm":
        norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
        return torch.stack([norm, torch.minimum(MAX_NORM / (norm + 1e-6), torch.ones_like(norm))])
    eight = case["state"] == "e4m3"
    t, lay = s["step"] + 1, s["layout"]
    m, v = s["m"], s["v"]
    if eight:
        m = (m.view(torch.float8_e4m3fn).double().view(-1, BLOCK) * s["m_scales"].double()[:, None]).view(-1)
        v = (v.view(torch.float8_e4m3fn).double().view(-1, BLOCK) * s["v_scales"].double()[:, None]).view(-1)
    g = s["grads"].double() * s["clip"].double()
    m = BETA1 * m.double() + (1 - BETA1) * g
    v = BETA2 * v.double() + (1 - BETA2) * g.square()
    del g
    p = s["params"].double()
    p[:lay.split] *= 1 - LR * DECAY
    p -= LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    out = {"params": p, "m": m, "v": v}
    if eight:
        r = _random_numbers(dict(s, step=t)).double()
        for name, x in (("m", m), ("v", v)):
            out[name], out[name + "_scales"] = _exact_codes(x.view(-1, BLOCK), r, name == "v")
            out[name] = out[name].view(-1)
    if s["copy"] is not None:
        out["copy"] = p
    return out
