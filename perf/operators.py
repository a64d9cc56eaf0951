"""Timed cases of two operators on dense rows of logits: sampling with each sequence's own truncation
(`Context.sample`) and distillation from a teacher's top entries (`Context.distill`), with their plain
forms in elementary torch operations.

Inputs follow the recipe of `gen/` with the Zipf rank of an entry drawn uniformly from 1 .. V instead of
being its place in a permutation, which makes them quick to produce.
"""
import math

import torch

own = False

CHUNK = 1024            # vocabulary entries per chunk of the two-level draw
V_RANGE, B_RANGE, K_RANGE, ROWS_RANGE = (8000, 262144), (1, 512), (1, 1024), (1, 2048)


def listed():
    def sample(name, B, R, V, dtype, law, pad=0):
        return {"name": name, "kind": "sample", "B": B, "R": R, "V": V, "dtype": dtype, "law": law, "pad": pad}

    def distill(name, B, R, V, dtype, k, tail, grad, padded=0.0, pad=0):
        return {"name": name, "kind": "distill", "B": B, "R": R, "V": V, "dtype": dtype, "k": k, "tail": tail,
                "grad": grad, "padded": padded, "pad": pad}

    return [
        # one interactive sequence with a small vocabulary, top-k: latency
        sample("sample_1x1_v32000_f32_k", 1, 1, 32000, "f32", "k"),
        # a small serving batch, nucleus and min-p together
        sample("sample_8x1_v128256_bf16_p_minp", 8, 1, 128256, "bf16", "p_minp"),
        # a full batch whose requests each bring their own truncation, some none at all
        sample("sample_256x1_v128256_bf16_mixed", 256, 1, 128256, "bf16", "mixed"),
        # several positions a sequence, temperature alone: no truncation
        sample("sample_64x4_v151936_bf16_plain", 64, 4, 151936, "bf16", "plain"),
        # an odd vocabulary in padded rows of a model head that leaves fp32
        sample("sample_24x4_v50381_f32_k_p", 24, 4, 50381, "f32", "k_p", 3),
        # the largest vocabulary, a full batch, nucleus
        sample("sample_512x1_v262144_bf16_p", 512, 1, 262144, "bf16", "p"),
        # the smallest training step: one draft of four positions
        distill("distill_1x4_v32000_f32_k32", 1, 4, 32000, "f32", 32, False, True),
        # the loss alone, as an evaluation has it, for a batch of drafts
        distill("distill_8x5_v128256_bf16_k64_eval", 8, 5, 128256, "bf16", 64, False, False),
        # a training batch of two sequences of 1024 positions, renormalised rows
        distill("distill_2x1024_v128256_bf16_k64", 2, 1024, 128256, "bf16", 64, False, True),
        # drafts of eight positions against raw probabilities: the rest of the teacher's mass counts
        distill("distill_64x8_v151936_bf16_k128_tail", 64, 8, 151936, "bf16", 128, True, True),
        # an odd vocabulary, a third of the positions padding
        distill("distill_3x333_v50381_bf16_k50_tail_padded", 3, 333, 50381, "bf16", 50, True, True, 0.33),
        # the widest sparse rows on the largest vocabulary, fp32 logits
        distill("distill_4x64_v262144_f32_k1024", 4, 64, 262144, "f32", 1024, False, True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    while True:
        V, dtype = log_int(*V_RANGE), rng.choice(["bf16", "bf16", "f32"])
        pad = rng.choice([0, 0, 0, 8, rng.randrange(1, 64)])
        if rng.random() < 0.5:
            case = {"kind": "sample", "B": log_int(*B_RANGE), "R": rng.choice([1, 1, 1, 2, 5]), "V": V, "dtype": dtype,
                    "law": rng.choice(["k", "p", "k_p", "p_minp", "minp", "plain", "mixed"]), "pad": pad}
        else:
            rows = log_int(*ROWS_RANGE)
            B = min(rows, log_int(1, 64))
            case = {"kind": "distill", "B": B, "R": max(1, rows // B), "V": V, "dtype": dtype,
                    "k": min(log_int(*K_RANGE), V), "tail": rng.random() < 0.5, "grad": rng.random() < 0.75,
                    "padded": rng.choice([0.0, 0.0, 0.25]), "pad": pad}
        most = max(work(c)["bytes"] for c in listed() if c["kind"] == case["kind"])
        if work(case)["bytes"] <= most:
            return case


def work(case):
    rows = case["B"] * case["R"]
    row = case["V"] * (2 if case["dtype"] == "bf16" else 4)
    if case["kind"] == "sample":
        # a row, its temperature and truncation, two uniforms; token, probability, log-probability, count.
        # An exponential, a multiplication and an addition an entry.
        return {"bytes": rows * (row + 8 + 16) + case["B"] * 16, "flops": 3 * rows * case["V"]}
    read = rows * (1 - case["padded"])
    return {"bytes": read * (row + 8 * case["k"]) + rows * (12 + (row if case["grad"] else 0)) + case["B"] * 4,
            "flops": (6 if case["grad"] else 3) * read * case["V"]}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _base(case, g):
    B, R, V = case["B"], case["R"], case["V"]
    base = torch.rand((B, R, V), generator=g, device="cuda").mul_(V - 1).add_(1).log_().mul_(-1.1)
    return base.add_(_normal((B, R, V), g), alpha=1.5)


def _stored(values, case):
    """`values` [B, R, V] in the case's type, in rows of V + pad elements."""
    B, R, V = values.shape
    buf = torch.empty((B, R, V + case["pad"]), dtype=_dtype(case), device="cuda")
    buf[..., V:] = float("nan")
    buf[..., :V] = values
    return buf[..., :V]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, R, V = case["B"], case["R"], case["V"]
    base = _base(case, g)
    temperature = 0.5 + 0.7 * torch.rand((B,), generator=g, device="cuda")
    state = {"case": case, "temperature": temperature, "context": None}

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if case["kind"] == "sample":
        state["logits"] = _stored(base, case)
        state["u"] = rand(B, R, 2).clamp_(max=1 - 2.0 ** -24)
        law = case["law"]
        k = (16 * 64 ** rand(B)).to(torch.int32)                 # 16 .. 1023
        p, m = 0.8 + 0.19 * rand(B), 0.002 + 0.1 * rand(B)
        if law == "mixed":                                      # each limit on for about half of the requests
            on = rand(3, B) < 0.5
            k, p, m = torch.where(on[0], k, 0), torch.where(on[1], p, 1.0), torch.where(on[2], m, 0.0)
        state["top_k"] = k if law in ("k", "k_p", "mixed") else None
        state["top_p"] = p if law in ("p", "k_p", "p_minp", "mixed") else None
        state["min_p"] = m if law in ("minp", "p_minp", "mixed") else None
        return _with_context(state, case, 1)

    # the student is the teacher of the recipe with noise on top, at the same temperature
    K = case["k"]
    state["logits"] = _stored(0.8 * base + _normal((B, R, V), g), case)
    top, idx = base.topk(K, dim=-1)
    z = (base / temperature[:, None, None]).logsumexp(-1, keepdim=True)
    prob = (top / temperature[:, None, None] - z).exp()
    if not case["tail"]:
        prob = prob / prob.sum(-1, keepdim=True)
    count = torch.full((B, R), K, dtype=torch.int32, device="cuda")
    if case["padded"]:
        count[rand(B, R) < case["padded"]] = 0
    behind = torch.arange(K, device="cuda") >= count[..., None]
    state["t_idx"] = torch.where(behind, -1, idx).to(torch.int32)
    state["t_prob"] = torch.where(behind, 0.0, prob)
    state["t_count"] = count
    state["weight"] = (count > 0).float() / (count > 0).sum().clamp(min=1)      # the mean over the positions that count
    return _with_context(state, case, K)


def _with_context(state, case, k):
    if own:
        import paper_2603_19133_b200 as ps
        state["context"] = ps.Context(1, 1, case["V"], k)
    return state


def run(state):
    case = state["case"]
    if own:
        ctx = state["context"]
        if case["kind"] == "sample":
            token, prob, logprob, count = ctx.sample(state["logits"], state["temperature"], state["u"], state["top_k"],
                                                     state["top_p"], state["min_p"])
            return {"token": token, "prob": prob, "logprob": logprob, "count": count}
        loss, grad = ctx.distill(state["logits"], state["temperature"], state["t_idx"], state["t_prob"], state["t_count"],
                                 weight=state["weight"], tail=case["tail"], want_grad=case["grad"])
        return {"loss": loss, "grad": grad} if case["grad"] else {"loss": loss}
    return _plain_sample(state) if case["kind"] == "sample" else _plain_distill(state)


def _plain_sample(state):
    # In 64 bits: which entries are kept and drawn is decided next to borders that 32 bits move.
    logits, u = state["logits"].float(), state["u"].double()
    B, R, V = logits.shape
    T = state["temperature"].double()[:, None, None]
    value, order = torch.sort(logits, dim=-1, descending=True, stable=True)
    w = torch.exp(value.double() / T - value[..., :1].double() / T)
    Z = w.sum(-1, keepdim=True)
    kept = value > -math.inf
    if state["top_k"] is not None:
        k = state["top_k"][:, None, None]
        kept &= (k == 0) | (torch.arange(V, device=logits.device) < k)
    if state["top_p"] is not None:
        p = state["top_p"].double()[:, None, None]
        before = torch.cumsum(w, -1).roll(1, -1)
        before[..., 0] = 0.0
        kept &= (p >= 1) | (before < p * Z)
        del before
    if state["min_p"] is not None:
        kept &= w >= state["min_p"].double()[:, None, None]
    count = kept.sum(-1, dtype=torch.int32)
    w = torch.zeros_like(w).scatter_(-1, order, w * kept)       # in the order of the vocabulary, 0 where not kept
    del order, value, kept
    chunks = torch.nn.functional.pad(w, (0, -V % CHUNK)).view(B, R, -1, CHUNK)
    upto = torch.cumsum(chunks.sum(-1), -1)
    W = upto[..., -1:]
    chunk = (upto <= u[..., :1] * W).sum(-1, keepdim=True).clamp(max=upto.shape[-1] - 1)
    inside = torch.cumsum(chunks.gather(2, chunk[..., None].expand(B, R, 1, CHUNK))[:, :, 0], -1)
    entry = (inside <= u[..., 1:] * inside[..., -1:]).sum(-1, keepdim=True).clamp(max=CHUNK - 1)
    token = chunk * CHUNK + entry
    weight = w.gather(-1, token)
    return {"token": token[..., 0].to(torch.int32), "prob": (weight / W)[..., 0].float(),
            "logprob": torch.log(weight / Z)[..., 0].float(), "count": count}


def _plain_distill(state):
    case, logits = state["case"], state["logits"]
    K, V = case["k"], logits.shape[-1]
    T = state["temperature"][:, None, None]
    x = logits.float() / T
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    valid = torch.arange(K, device=x.device) < state["t_count"][..., None]
    idx = torch.where(valid, state["t_idx"], 0).long()
    # the teacher's sums and their complement in 64 bits: 1 - sum of nearly everything
    t = torch.where(valid, state["t_prob"], 0.0).double()
    A = t.sum(-1, keepdim=True)
    t_log_t = torch.where(t > 0, t * torch.log(t.clamp(min=1e-300)), 0.0)
    log_s = (x.gather(-1, idx) - m - torch.log(total)).double()
    loss = (t_log_t - torch.where(t > 0, t * log_s, 0.0)).sum(-1, keepdim=True)
    outside = torch.zeros_like(x).scatter_add_(-1, idx, valid.float()) == 0
    scale = A
    if case["tail"]:
        r = (1 - A).clamp(min=0) * (state["t_count"][..., None] > 0)
        rest = (e * outside).sum(-1, keepdim=True)
        loss = loss + torch.where(r > 0, r * (torch.log(r.clamp(min=1e-300)) - torch.log(rest / total).double()), 0.0)
        scale = A + r
    loss = loss[..., 0].float()
    if not case["grad"]:
        return {"loss": loss}
    s = e.div_(total)
    del x
    target = torch.zeros_like(s).scatter_add_(-1, idx, t.float())
    grad = scale.float() * s - target
    if case["tail"]:
        grad = grad - outside * s * (r * (total / rest)).float()
    grad = grad * (state["weight"][..., None] / T)
    return {"loss": loss, "grad": grad.to(logits.dtype)}


def exact(case, seed):
    """The definitions in 64 bits, a row at a time."""
    state = prepare(case, seed)
    B, R, V = case["B"], case["R"], case["V"]
    if case["kind"] == "sample":
        out = {"token": torch.empty((B, R), dtype=torch.int32, device="cuda"),
               "prob": torch.empty((B, R), dtype=torch.float64, device="cuda"),
               "logprob": torch.empty((B, R), dtype=torch.float64, device="cuda"),
               "count": torch.empty((B, R), dtype=torch.int32, device="cuda")}
        for b in range(B):
            for i in range(R):
                limits = [None if state[n] is None else state[n][b].double() for n in ("top_k", "top_p", "min_p")]
                _exact_draw(state["logits"][b, i].double(), state["temperature"][b].double(), limits,
                            state["u"][b, i].double(), {n: v[b, i] for n, v in out.items()})
        return out
    out = {"loss": torch.zeros((B, R), dtype=torch.float64, device="cuda")}
    if case["grad"]:
        out["grad"] = torch.zeros((B, R, V), dtype=torch.float64, device="cuda")
    counts = state["t_count"].tolist()
    for b in range(B):
        for i in range(R):
            n = counts[b][i]
            if n == 0:
                continue
            T = state["temperature"][b].double()
            logs = torch.log_softmax(state["logits"][b, i].double() / T, 0)
            at, t = state["t_idx"][b, i, :n].long(), state["t_prob"][b, i, :n].double()
            loss = torch.special.xlogy(t, t).sum() - (t * logs[at]).sum()
            grad = t.sum() * logs.exp()
            grad[at] -= t
            if case["tail"]:
                r = (1 - t.sum()).clamp(min=0)
                rest = logs.clone()
                rest[at] = -math.inf
                log_rest = torch.logsumexp(rest, 0)
                loss = loss + torch.special.xlogy(r, r) - r * log_rest
                grad = grad + r * logs.exp() - r * (rest - log_rest).exp()
            out["loss"][b, i] = loss
            if case["grad"]:
                out["grad"][b, i] = grad * state["weight"][b, i].double() / T
    return out


def _exact_draw(l, T, limits, u, out):
    top_k, top_p, min_p = limits
    logp = torch.log_softmax(l / T, 0)
    p = logp.exp()
    order = torch.argsort(l, descending=True, stable=True)
    sorted_p = p[order]
    n = torch.isfinite(l).sum()
    if top_k is not None:
        n = torch.where(top_k > 0, torch.minimum(n, top_k.long()), n)
    if top_p is not None:
        reach = (torch.cumsum(sorted_p, 0) < top_p * sorted_p.sum()).sum() + 1
        n = torch.where(top_p < 1, torch.minimum(n, reach), n)
    if min_p is not None:
        n = torch.minimum(n, (torch.exp((l - l.max()) / T) >= min_p).sum())
    q = torch.zeros_like(p)
    q[order] = torch.where(torch.arange(l.numel(), device=l.device) < n, sorted_p, 0.0)
    W = q.sum()
    mass = torch.stack([c.sum() for c in q.split(CHUNK)])
    c = torch.searchsorted(torch.cumsum(mass, 0), (u[0] * W).reshape(1), right=True)[0]
    part = q.new_zeros(CHUNK)
    at = c * CHUNK + torch.arange(CHUNK, device=l.device)
    part = torch.where(at < l.numel(), q[at.clamp(max=l.numel() - 1)], part)
    e = torch.searchsorted(torch.cumsum(part, 0), (u[1] * mass[c]).reshape(1), right=True)[0]
    token = c * CHUNK + e
    out["token"].copy_(token)
    out["prob"].copy_(q[token] / W)
    out["logprob"].copy_(logp[token])
    out["count"].copy_(n)
