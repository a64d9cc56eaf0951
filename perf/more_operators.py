"""Timed cases of the operators around a draft-and-verify step, with their plain forms in elementary torch operations: penalties for
repeated tokens, biases and grammar masks on rows of logits (`Context.penalize`) and their gradient (`Context.penalize_grad`),
the tokens that a step leaves put behind each sequence's history (`Context.append`), and the global norm and clipping of the
gradients of a drafter in training (`Context.grad_norm`, `Context.clip_grad`).
"""
import math

import torch

own = False

V_RANGE, B_RANGE, L_RANGE, K_RANGE = (8000, 262144), (1, 512), (1, 131072), (1, 300)
D_RANGE = (16, 2048)            # width of a drafter
MOST_TOKENS = 1 << 23           # tokens of history in one case
MASK_STATES = 64                # grammar states whose masks are kept


def listed():
    def rules(name, B, R, V, dtype, length, law, k=0, mask="none", pad=0, inplace=False):
        return {"name": name, "kind": "rules", "B": B, "R": R, "V": V, "dtype": dtype, "length": length, "law": law, "k": k,
                "mask": mask, "pad": pad, "inplace": inplace}

    def grad(name, B, R, V, dtype, length, law, mask="none", pad=0):
        return {"name": name, "kind": "rules_grad", "B": B, "R": R, "V": V, "dtype": dtype, "length": length, "law": law, "k": 0,
                "mask": mask, "pad": pad, "inplace": False}

    def append(name, B, G, L):
        return {"name": name, "kind": "append", "B": B, "G": G, "L": L}

    def clip(name, d, layers, V, dtype, what):
        return {"name": name, "kind": "clip", "d": d, "layers": layers, "V": V, "dtype": dtype, "what": what}

    return [
        # one interactive sequence, a short conversation, the repetition penalty alone: latency
        rules("rules_1x1_v32000_f32_rep", 1, 1, 32000, "f32", 500, "rep"),
        # a small serving batch of drafts over long documents with every rule on: the history is as large as a row
        rules("rules_8x6_v128256_bf16_long", 8, 6, 128256, "bf16", 100000, "all", 64, "mixed"),
        # the target rows of a full batch before they are verified: the three penalties
        rules("rules_256x7_v128256_bf16_pen", 256, 7, 128256, "bf16", 4000, "pen"),
        # an odd vocabulary in padded rows, every rule, up to 300 biases
        rules("rules_24x5_v50381_f32_all", 24, 5, 50381, "f32", 2000, "all", 300, "mixed", 3),
        # structured output for the largest vocabulary, a token at a time: grammar masks alone, in place
        rules("rules_512x1_v262144_bf16_mask", 512, 1, 262144, "bf16", 0, "mask", 0, "mixed", 0, True),
        # training of a drafter on positions that were drawn under rules: drafts of eight positions
        grad("rules_grad_64x8_v151936_bf16_all", 64, 8, 151936, "bf16", 2000, "all", "mixed"),
        # the same over whole texts: every position has the tokens before it in its history
        grad("rules_grad_2x333_v50381_f32_rep", 2, 333, 50381, "f32", 64, "rep", "none", 0),
        # a single sequence after its draft of four was verified
        append("append_1x4_l4096", 1, 4, 4096),
        # a full batch after drafts of eight
        append("append_512x8_l16384", 512, 8, 16384),
        # the gradient of a small drafter, fp32: its norm, and the gradients clipped
        clip("clip_d256_2layers_v1000_f32", 256, 2, 1000, "f32", "clip"),
        # an ordinary drafter whose gradient stays below the limit: nothing to write
        clip("clip_d1024_4layers_v32000_mixed_within", 1024, 4, 32000, "mixed", "within"),
        # a wide drafter with its own embedding and head, bf16
        clip("clip_d2048_2layers_v128256_bf16", 2048, 2, 128256, "bf16", "clip"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    while True:
        kind = rng.choice(["rules", "rules", "rules_grad", "append", "clip", "clip"])
        if kind == "append":
            case = {"kind": kind, "B": log_int(*B_RANGE), "G": rng.randint(0, 16), "L": log_int(64, L_RANGE[1])}
            if case["B"] * case["L"] > MOST_TOKENS:
                continue
        elif kind == "clip":
            case = {"kind": kind, "d": log_int(*D_RANGE), "layers": rng.randint(1, 6), "V": log_int(100, 128256),
                    "dtype": rng.choice(["bf16", "f32", "mixed"]), "what": rng.choice(["norm", "clip", "clip", "within"])}
        else:
            law = rng.choice(["rep", "freq", "pen", "all", "all", "mask"])
            rows, B = log_int(1, 2048), log_int(*B_RANGE)
            R = rng.choice([1, 1, 2, 5, 9]) if kind == "rules" else max(1, rows // B)
            case = {"kind": kind, "B": B, "R": R, "V": log_int(*V_RANGE), "dtype": rng.choice(["bf16", "bf16", "f32"]),
                    "length": 0 if law == "mask" else log_int(*L_RANGE), "law": law,
                    "k": log_int(*K_RANGE) if law == "all" and kind == "rules" else 0,
                    "mask": "mixed" if law == "mask" else rng.choice(["none", "mixed"]) if law == "all" else "none",
                    "pad": rng.choice([0, 0, 0, 8, rng.randrange(1, 64)]), "inplace": law == "mask" and kind == "rules"}
            if B * max(case["length"], R) > MOST_TOKENS:
                continue
        if work(case)["bytes"] <= max(work(c)["bytes"] for c in listed() if c["kind"] == kind):
            return case


# ---- inputs ----------------------------------------------------------------------------------

def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


def _tokens(shape, V, g):
    """Token ids as text has them: frequent ones come first in a vocabulary."""
    return torch.rand(shape, generator=g, device="cuda").mul_(math.log(V)).exp_().sub_(1).to(torch.int32).clamp_(0, V - 1)


def _shapes(case):
    """The parameters of a small decoder: (shape, whether it is kept in fp32 among bf16 ones)."""
    d, f, V = case["d"], 4 * case["d"], case["V"]
    shapes = [((V, d), False)]
    for _ in range(case["layers"]):
        shapes += [((d,), True), ((d + 2 * max(1, d // 4), d), False), ((d, d), False), ((d,), True), ((2 * f, d), False), ((d, f), False)]
    return shapes + [((d,), True), ((V, d), False)]


def _grad_type(case, small):
    return _dtype("f32" if case["dtype"] == "f32" or (case["dtype"] == "mixed" and small) else "bf16")


def _stored(values, case):
    """`values` [B, R, V] in the case's type, in rows of V + pad elements."""
    B, R, V = values.shape
    buf = torch.empty((B, R, V + case["pad"]), dtype=_dtype(case["dtype"]), device="cuda")
    buf[..., V:] = float("nan")
    buf[..., :V] = values
    return buf[..., :V]


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _masks(case, g):
    """Masks of grammar states, 32 entries a word: every other state allows a few tokens (the next is a bracket, a digit), the others
    all but a few (inside a text).  A fifth of the rows is free of a grammar."""
    B, R, V = case["B"], case["R"], case["V"]
    M = min(B * R, MASK_STATES)
    few = torch.rand((M, V), generator=g, device="cuda")
    odd = (torch.arange(M, device="cuda") % 2 == 1)[:, None]
    allowed = torch.where(odd, few < 0.97, few < 40 / V)
    allowed[:, 0] = True
    allowed = torch.nn.functional.pad(allowed, (0, -V % 32)).view(M, -1, 32).long()
    words = (allowed << torch.arange(32, device="cuda")).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).contiguous()
    row = torch.arange(B * R, device="cuda").view(B, R) % (M + max(1, M // 4))
    return words, torch.where(row < M, row, -1).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case, "context": None}
    if case["kind"] == "clip":
        state["grads"] = []
        for shape, small in _shapes(case):
            t = torch.randn(shape, generator=g, device="cuda", dtype=_grad_type(case, small))
            scale = 10.0 ** (-6 + 4 * torch.rand((1,), generator=g, device="cuda"))
            if shape[0] == case["V"] and not state["grads"]:            # the embedding: tokens that did not occur have none
                scale = scale * (torch.rand((shape[0], 1), generator=g, device="cuda") < 0.3)
            state["grads"].append(t.mul_(scale.to(t.dtype)))
        total = math.sqrt(sum(float(t.float().square().sum(dtype=torch.float64)) for t in state["grads"]))
        state["max_norm"] = total * (2.0 if case["what"] == "within" else 0.25)
        state["out"] = [torch.empty_like(t) for t in state["grads"]] if case["what"] == "clip" else None
        return _with_context(state, 1024)
    B = case["B"]

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if case["kind"] == "append":
        G, L = case["G"], case["L"]
        state["history"] = _tokens((B, L), 32000, g)
        state["length"] = (rand(B) * (L - G)).to(torch.int32)           # (room for G + 1 tokens)
        state["draft_tok"] = _tokens((B, G), 32000, g) if G else None
        state["accept_len"] = (rand(B) * (G + 1)).to(torch.int32).clamp_(max=G) if G else None
        state["token"] = _tokens((B,), 32000, g)
        return _with_context(state, 32000)

    R, V, L, law = case["R"], case["V"], case["length"], case["law"]
    base = rand(B, R, V).mul_(V - 1).add_(1).log_().mul_(-1.1).add_(_normal((B, R, V), g), alpha=1.5)
    state["logits"] = _stored(base, case)
    if case["kind"] == "rules_grad":
        state["grad"] = _normal((B, R, V), g).mul_(1e-3).to(_dtype(case["dtype"]))
    for name in ("history", "length", "prompt_length", "draft_tok", "repetition", "presence", "frequency", "bias", "mask", "mask_row"):
        state[name] = None
    if law != "mask":
        state["history"] = _tokens((B, L), V, g)
        length = (rand(B) * (L + 1)).to(torch.int32).clamp_(max=L)
        length[B // 2] = L
        state["length"] = length
        state["prompt_length"] = (rand(B) * (length + 1)).to(torch.int32).clamp_(max=L)
        state["prompt_length"] = torch.minimum(state["prompt_length"], length)
        state["draft_tok"] = _tokens((B, R - 1), V, g) if R > 1 else None
    on = rand(3, B) < 0.75                                              # a quarter of the requests leaves each penalty off
    if law in ("rep", "pen", "all"):
        state["repetition"] = torch.where(on[0], 1 + 0.3 * rand(B), 1.0)
    if law in ("freq", "pen", "all"):
        state["presence"] = torch.where(on[1], 1.5 * rand(B) - 0.3, 0.0)
        state["frequency"] = torch.where(on[2], rand(B) - 0.2, 0.0)
    if case["k"]:
        K = min(case["k"], V)
        idx = (torch.arange(K, device="cuda") * (V // K) + (rand(B, K) * (V // K)).long().clamp(max=V // K - 1)).to(torch.int32)
        state["bias"] = (idx.contiguous(), 8 * _normal((B, K), g), (rand(B) * (K + 1)).to(torch.int32).clamp_(max=K))
    if case["mask"] != "none":
        state["mask"], state["mask_row"] = _masks(case, g)
    return _with_context(state, V)


def _with_context(state, V):
    if own:
        import paper_2603_19133_b200 as ps
        state["context"] = ps.Context(1, 1, V, 1)
    return state


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    if case["kind"] == "append":
        # on average half of a draft and one more token are copied; length and count in, length out
        return {"bytes": case["B"] * (8 * (case["G"] / 2 + 1) + 12), "flops": 0}
    if case["kind"] == "clip":
        n = [math.prod(shape) for shape, _ in _shapes(case)]
        size = sum(k * (2 if _grad_type(case, small) == torch.bfloat16 else 4) for k, (_, small) in zip(n, _shapes(case)))
        return {"bytes": size * (2 if case["what"] == "clip" else 1) + 4, "flops": (3 if case["what"] == "clip" else 2) * sum(n)}
    B, R, V, rows = case["B"], case["R"], case["V"], case["B"] * case["R"]
    row, words = V * _size(case["dtype"]), 4 * -(-V // 32)
    M = min(rows, MASK_STATES)
    # rows whose grammar allows few tokens: their entries are written, not read
    tight = loose = 0.0
    if case["mask"] != "none":
        period = M + max(1, M // 4)
        tight, loose = rows * -(-M // 2) / period, rows * (M // 2) / period
    side = B * (case["length"] / 2 + R) * 4 + B * case["k"] / 2 * 8 + B * 20 + min(rows, M) * words * (case["mask"] != "none")
    if case["inplace"]:
        return {"bytes": tight * row + loose * 0.03 * row + side, "flops": 0}
    read = rows - tight
    if case["kind"] == "rules_grad" and case["law"] in ("rep", "pen", "all"):
        side += B * R * min(case["length"] / 2, V / 4) * _size(case["dtype"])     # the sign of the logits of the tokens seen
    return {"bytes": (read + rows) * row + side, "flops": rows * min(case["length"] / 2, V / 4) * 4}


# ---- one pass ----------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if not own:
        return {"append": _plain_append, "clip": _plain_clip, "rules": _plain_rules, "rules_grad": _plain_rules}[case["kind"]](state)
    ctx = state["context"]
    if case["kind"] == "append":
        length = ctx.append(state["history"], state["length"], state["token"], state["draft_tok"], state["accept_len"])
        return {"history": state["history"], "length": length}
    if case["kind"] == "clip":
        if case["what"] == "norm":
            return {"norm": ctx.grad_norm(state["grads"])}
        norm = ctx.clip_grad(state["grads"], state["max_norm"], out=state["out"])
        return {"norm": norm, "grads": state["out"] or state["grads"]}
    rules = {n: state[n] for n in ("history", "length", "prompt_length", "draft_tok", "repetition", "presence", "frequency", "bias",
                                   "mask", "mask_row")}
    if case["kind"] == "rules":
        return {"logits": ctx.penalize(state["logits"], **rules, out=state["logits"] if case["inplace"] else None)}
    return {"grad": ctx.penalize_grad(state["grad"], state["logits"], **rules)}


def _plain_append(state):
    history, length = state["history"], state["length"]
    if state["draft_tok"] is None:
        history.scatter_(1, length[:, None].long(), state["token"][:, None])
        return {"history": history, "length": length + 1}
    G, n = state["draft_tok"].shape[1], state["accept_len"]
    j = torch.arange(G + 1, device=history.device)
    new = torch.cat([state["draft_tok"], state["token"][:, None]], 1)
    new = torch.where(j == n[:, None], state["token"][:, None], new)
    at = (length[:, None] + j).long()                   # (there is room for a whole draft and one more token)
    history.scatter_(1, at, torch.where(j <= n[:, None], new, history.gather(1, at)))
    return {"history": history, "length": length + n + 1}


def _plain_clip(state):
    grads, what = state["grads"], state["case"]["what"]
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum().sqrt()
    if what == "norm":
        return {"norm": norm.float().view(1)}
    scale = torch.where(norm > state["max_norm"], state["max_norm"] / norm, 1.0).float()
    if what == "within":
        for g in grads:
            g.copy_((g.float() * scale).to(g.dtype))
        return {"norm": norm.float().view(1), "grads": grads}
    for o, g in zip(state["out"], grads):
        o.copy_((g.float() * scale).to(g.dtype))
    return {"norm": norm.float().view(1), "grads": state["out"]}


def _allowed(state, rows, V):
    """The rows' masks [.., V], true where a token may come; rows without one allow all."""
    words = state["mask"][rows.long().clamp(min=0)]
    bits = (words[..., None] >> torch.arange(32, device=words.device)) & 1
    return (bits.flatten(-2)[..., :V] != 0) | (rows < 0)[..., None]


def _plain_rules(state):
    case, logits = state["case"], state["logits"]
    B, R, V = logits.shape
    if case["inplace"]:
        logits.masked_fill_(~_allowed(state, state["mask_row"], V), -math.inf)
        return {"logits": logits}
    backward = case["kind"] == "rules_grad"
    source = state["grad"] if backward else logits
    out = torch.empty((B, R, V), dtype=logits.dtype, device=logits.device)
    seen = count = None
    if state["history"] is not None:
        at = torch.arange(state["history"].shape[1], device=logits.device)
        valid = at < state["length"][:, None]
        made = valid & (at >= state["prompt_length"][:, None])
        token = state["history"].long()
        seen = torch.zeros((B, V), dtype=torch.int32, device=logits.device).scatter_add_(1, token, valid.int())
        count = torch.zeros((B, V), dtype=torch.int32, device=logits.device).scatter_add_(1, token, made.int())
    for i in range(R):
        if i and seen is not None:
            drafted = state["draft_tok"][:, i - 1:i].long()
            one = torch.ones_like(drafted, dtype=torch.int32)
            seen.scatter_add_(1, drafted, one)
            count.scatter_add_(1, drafted, one)
        x = source[:, i].float()
        if state["repetition"] is not None:
            rho = state["repetition"][:, None]
            l = logits[:, i]
            x = torch.where(seen > 0, torch.where(l > 0, x / rho, x * rho), x)
        if not backward:
            if state["frequency"] is not None:
                x = x - state["frequency"][:, None] * count
            if state["presence"] is not None:
                x = x - state["presence"][:, None] * (count > 0)
            if state["bias"] is not None:
                idx, value, n = state["bias"]
                given = torch.arange(idx.shape[1], device=x.device) < n[:, None]
                x = x.scatter_add(1, idx.long(), torch.where(given, value, 0.0))
        if state["mask"] is not None:
            x = x.masked_fill(~_allowed(state, state["mask_row"][:, i], V), 0.0 if backward else -math.inf)
        out[:, i] = x.to(out.dtype)
    return {"grad" if backward else "logits": out}


def exact(case, seed):
    """The definitions in 64 bits, a sequence and a row at a time."""
    state = prepare(case, seed)
    if case["kind"] == "append":
        history, length = state["history"].tolist(), state["length"].tolist()
        draft = state["draft_tok"].tolist() if case["G"] else [[]] * case["B"]
        taken = state["accept_len"].tolist() if case["G"] else [0] * case["B"]
        for b, last in enumerate(state["token"].tolist()):
            new = draft[b][:taken[b]] + [last]
            history[b][length[b]:length[b] + len(new)] = new
            length[b] += len(new)
        return {"history": torch.tensor(history, dtype=torch.int32), "length": torch.tensor(length, dtype=torch.int32)}
    if case["kind"] == "clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t.double()) for t in state["grads"]]))
        if case["what"] == "norm":
            return {"norm": norm.view(1)}
        factor = min(1.0, state["max_norm"] / float(norm))
        return {"norm": norm.view(1), "grads": [t.double() * factor for t in state["grads"]]}
    B, R, V = state["logits"].shape
    backward = case["kind"] == "rules_grad"
    out = torch.empty((B, R, V), dtype=torch.float64, device="cuda")
    for b in range(B):
        before = made = None
        if state["history"] is not None:
            n, p = int(state["length"][b]), int(state["prompt_length"][b])
            before = torch.bincount(state["history"][b, :p].long(), minlength=V) > 0
            made = torch.bincount(state["history"][b, p:n].long(), minlength=V)
        for i in range(R):
            if made is not None and i:
                made[state["draft_tok"][b, i - 1].long()] += 1
            l = state["logits"][b, i].double()
            factor, shift = torch.ones_like(l), torch.zeros_like(l)
            if state["repetition"] is not None:
                rho = state["repetition"][b].double()
                factor[before | (made > 0)] = rho
                factor = torch.where(l > 0, 1 / factor, factor)
            if state["frequency"] is not None:
                shift += state["frequency"][b].double() * made + state["presence"][b].double() * made.clamp(max=1)
            y = factor * state["grad"][b, i].double() if backward else factor * l - shift
            if state["bias"] is not None and not backward:
                k = int(state["bias"][2][b])
                y[state["bias"][0][b, :k].long()] += state["bias"][1][b, :k].double()
            if state["mask"] is not None and int(state["mask_row"][b, i]) >= 0:
                v = torch.arange(V, device="cuda")
                word = state["mask"][int(state["mask_row"][b, i])][v // 32].long()
                y[(word >> (v % 32)) % 2 == 0] = 0.0 if backward else -math.inf
            out[b, i] = y
    return {"grad" if backward else "logits": out}
