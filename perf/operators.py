"""Cases of the head's losses: softmax cross entropy of tokens and distillation from a teacher's top logits, each with its
gradient, from the rows that feed the head and the head's weights.

`listed()` are the named cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a learner has in hand (the
rows, the head, the targets, and for a gradient the log-normalisers of the forward pass and the rows' coefficients), `run()` is one
call, in its plain form or (`own`) through the framework, `exact()` the same in 64 bits, `work()` the bytes and operations a call
cannot do without.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, loss, call, dtype, rows, d, vocab, top=0, temperature=0.0):
    return dict(name=name, loss=loss, call=call, dtype=dtype, rows=rows, d=d, vocab=vocab, top=top, temperature=temperature)


def listed():
    return [
        # the tiny float32 policy's chunk of one batch (4 x 7 action tokens over 256 bins): the smallest call, all latency
        _case("token loss f32 28x256 bins", "token", "loss", "f32", 28, 256, 256),
        # the same policy trained on its whole vocabulary, a ragged batch with its gradient
        _case("token grad f32 333x1024", "token", "grad", "f32", 333, 256, 1024),
        # learner step of the 7B policy on action bins: 64 observations x 7 tokens, coefficients of either sign
        _case("token grad 448x256 bins 7b", "token", "grad", "bf16", 448, 4096, 256, temperature=1.0),
        # one token over the whole vocabulary of the 7B model: the head is read once, nothing else counts
        _case("token loss 1x32000 7b", "token", "loss", "bf16", 1, 4096, 32000),
        # a chunk of 56 action tokens of one observation against the whole vocabulary
        _case("token grad 56x32000 7b", "token", "grad", "bf16", 56, 4096, 32000),
        # supervised start of the 12-layer model: an odd number of rows, a vocabulary with added tokens
        _case("token loss 2301x32003 small", "token", "loss", "bf16", 2301, 768, 32003),
        _case("token grad 1021x32003 small", "token", "grad", "bf16", 1021, 768, 32003),
        # supervised step of the 7B model: forward, and the largest call, its backward pass
        _case("token loss 8192x32000 7b", "token", "loss", "bf16", 8192, 4096, 32000),
        _case("token grad 8192x32000 7b", "token", "grad", "bf16", 8192, 4096, 32000),
        # distillation of a few rows from eight teacher logits each: latency
        _case("distill loss 7x32000 small top8", "distill", "loss", "bf16", 7, 768, 32000, 8, 1.5),
        # distillation of the 7B model: 64 teacher logits a row, some of them missing, rows without any
        _case("distill loss 4096x32000 7b top64", "distill", "loss", "bf16", 4096, 4096, 32000, 64, 2.0),
        _case("distill grad 2048x32000 7b top32", "distill", "grad", "bf16", 2048, 4096, 32000, 32, 1.0),
    ]


def draw(rng):
    """One more case: either loss, either direction, sizes log-uniform over the listed ranges, odd ones among them."""
    most = max(work(c)["flops"] for c in listed())

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        f32 = rng.random() < 0.25
        loss = rng.choice(["token", "distill"])
        c = dict(loss=loss, call=rng.choice(["loss", "grad"]), dtype="f32" if f32 else "bf16",
                 rows=log_int(1, 512 if f32 else 8192), d=log_int(8, 64) * 16 if f32 else log_int(2, 32) * 128,
                 vocab=log_int(200, 4096 if f32 else 33000), top=log_int(1, 100) if loss == "distill" else 0,
                 temperature=rng.choice([0.0, 1.0, round(rng.uniform(0.5, 2.0), 2)]))
        if work(c)["flops"] <= most:
            return c


# ---- inputs ---------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    """Rows of a final norm's scale, head rows of N(0, 0.02^2) as everywhere in the workloads; each row leans towards its target's
    head row by some nats, as a policy in training does.  One row in sixteen has no target (padding); its values are not
    finite, as memory nobody wrote may be."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed * 1000003 + case["rows"] * 31 + case["vocab"])
    T, d, V, k = case["rows"], case["d"], case["vocab"], case["top"]
    dt = DTYPES[case["dtype"]]

    def normal(*size):
        return torch.empty(size, device=DEVICE).normal_(0.0, 1.0, generator=gen)

    def ints(n, lo, hi):
        return torch.randint(lo, hi, (n,), device=DEVICE, generator=gen)

    head = normal(V, d).mul_(0.02).to(dt)
    labels = ints(T, 0, V)
    rows = normal(T, d)
    lean = torch.rand(T, 1, device=DEVICE, generator=gen) * (10.0 / (0.02 * 0.02 * d))      # up to ten nats
    rows = rows + lean * head[labels].float()
    idle = torch.rand(T, device=DEVICE, generator=gen) < 1.0 / 16
    idle[ints(1, 0, T)] = False
    rows[idle] = math.nan
    s = {"hidden": rows.to(dt), "head": head, "temperature": case["temperature"]}
    if case["loss"] == "token":
        s["labels"] = torch.where(idle, -100, labels).to(torch.int32)
    else:
        # k different ids a row, the label first; logits that fall off as a confident teacher's; a tenth of the entries missing
        step = 1 + (torch.rand(T, device=DEVICE, generator=gen) * max(1, (V - 1) // max(k, 1))).long().clamp(max=max(0, (V - 1) // max(k, 1) - 1))
        j = torch.arange(k, device=DEVICE)
        ids = (labels[:, None] + j[None, :] * step[:, None]) % V
        logits = 12.0 - 1.5 * torch.sqrt(j.float())[None, :] * (1.0 + 0.2 * normal(T, k).abs())
        gone = torch.rand(T, k, device=DEVICE, generator=gen) < 0.1
        gone[:, 0] = False
        gone |= idle[:, None]
        s["top_ids"] = torch.where(gone, -1, ids).to(torch.int32)
        s["top_logits"] = torch.where(gone, math.nan, logits)
    if case["call"] == "grad":
        # a mean over the rows that count, with coefficients of either sign (importance weight times advantage)
        s["grad_loss"] = torch.where(idle, 0.0, normal(T) / max(1, T))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["loss"], s["call"] = case["loss"], case["call"]
    if case["call"] == "grad":
        z = _logits(s, torch.float32)
        s["lse"] = torch.where(_has_target(s), _lse(z), 0.0)
    return s


# ---- plain form -----------------------------------------------------------------------------------------------
def _tau(s):
    return s["temperature"] if s["temperature"] > 0 else 1.0


def _has_target(s):
    V = s["head"].shape[0]
    if s["loss"] == "token":
        return (s["labels"] >= 0) & (s["labels"] < V)
    return ((s["top_ids"] >= 0) & (s["top_ids"] < V)).any(1)


def _rows(s, dt):
    """The rows, those without a target as zeros."""
    return torch.where(_has_target(s)[:, None], s["hidden"].to(dt), 0.0)


def _logits(s, dt):
    return _rows(s, dt) @ s["head"].to(dt).T / _tau(s)


def _lse(z):
    m = z.max(1).values
    return m + torch.log(torch.exp(z - m[:, None]).sum(1))


def _teacher(s, dt):
    """Probabilities of a row's teacher entries: a softmax over those that are there; ids of the others are 0, of probability 0."""
    V = s["head"].shape[0]
    there = (s["top_ids"] >= 0) & (s["top_ids"] < V)
    t = torch.where(there, s["top_logits"].to(dt) / _tau(s), -math.inf)
    m = t.max(1, keepdim=True).values
    e = torch.where(there, torch.exp(t - torch.where(m == -math.inf, 0.0, m)), 0.0)
    p = e / torch.where(there.any(1, keepdim=True), e.sum(1, keepdim=True), 1.0)
    return torch.where(there, s["top_ids"].long(), 0), p


def _plain(s):
    dt = torch.float32
    z = _logits(s, dt)
    live = _has_target(s)
    if s["call"] == "loss":
        lse = _lse(z)
        if s["loss"] == "token":
            y = torch.where(live, s["labels"].long(), 0)
            return {"loss": torch.where(live, lse - z.gather(1, y[:, None])[:, 0], 0.0), "lse": torch.where(live, lse, 0.0)}
        ids, p = _teacher(s, dt)
        logp = torch.log(torch.where(p > 0, p, 1.0))
        kl = (p * (logp - z.gather(1, ids) + lse[:, None])).sum(1)
        return {"loss": torch.where(live, kl, 0.0), "lse": torch.where(live, lse, 0.0)}
    dz = torch.exp(z - s["lse"][:, None])
    if s["loss"] == "token":
        y = torch.where(live, s["labels"].long(), 0)
        dz.scatter_add_(1, y[:, None], torch.full_like(dz[:, :1], -1.0))
    else:
        ids, p = _teacher(s, dt)
        dz.scatter_add_(1, ids, -p)
    dz = dz * (torch.where(live, s["grad_loss"], 0.0) / _tau(s))[:, None]
    out = s["hidden"].dtype
    return {"grad_hidden": (dz @ s["head"].to(dt)).to(out), "grad_head": (dz.T @ _rows(s, dt)).to(out)}


def run(state):
    if not own:
        return _plain(state)
    import paper_2603_18464_amd as P
    s = state
    if s["loss"] == "token":
        if s["call"] == "loss":
            loss, lse = P.token_loss(s["hidden"], s["head"], s["labels"], temperature=s["temperature"])
        else:
            gh, gw = P.token_loss_grad(s["hidden"], s["head"], s["labels"], s["lse"], s["grad_loss"], temperature=s["temperature"])
    else:
        if s["call"] == "loss":
            loss, lse = P.distill_loss(s["hidden"], s["head"], s["top_logits"], s["top_ids"], temperature=s["temperature"])
        else:
            gh, gw = P.distill_loss_grad(s["hidden"], s["head"], s["top_logits"], s["top_ids"], s["lse"], s["grad_loss"],
                                         temperature=s["temperature"])
    return {"loss": loss, "lse": lse} if s["call"] == "loss" else {"grad_hidden": gh, "grad_head": gw}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------
def exact(case, seed):
    """Row blocks: q = softmax of a row over the vocabulary, r = the target distribution (one token, or the teacher's over its
    entries), loss = sum r (log r - log q), gradient of the logits = coefficient (q - r) / temperature."""
    s = dict(_inputs(case, seed), loss=case["loss"], call=case["call"])
    tau = case["temperature"] or 1.0
    T, V, d = case["rows"], case["vocab"], case["d"]
    W = s["head"].double()
    H = s["hidden"].double()
    loss = torch.zeros(T, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros_like(loss)
    gh = torch.zeros(T, d, dtype=torch.float64, device=DEVICE) if case["call"] == "grad" else None
    gw = torch.zeros(V, d, dtype=torch.float64, device=DEVICE) if case["call"] == "grad" else None
    for t0 in range(0, T, 1024):
        t1 = min(T, t0 + 1024)
        r = torch.zeros(t1 - t0, V + 1, dtype=torch.float64, device=DEVICE)       # the last column takes what is not there
        if case["loss"] == "token":
            y = s["labels"][t0:t1].long()
            r.scatter_(1, torch.where((y < 0) | (y >= V), V, y)[:, None], 1.0)
        else:
            ids = s["top_ids"][t0:t1].long()
            out = (ids < 0) | (ids >= V)
            w = torch.exp(torch.where(out, -math.inf, (s["top_logits"][t0:t1].double() - 12.0) / tau))
            r.scatter_add_(1, torch.where(out, V, ids), w)
            r[:, V] = 0.0
            total = r.sum(1, keepdim=True)
            r = torch.where(total > 0, r / torch.where(total > 0, total, 1.0), 0.0)
        r = r[:, :V]
        live = r.sum(1) > 0
        h = H[t0:t1].masked_fill(~live[:, None], 0.0)
        z = (h @ W.T) / tau
        n = torch.logsumexp(z, 1)
        if case["call"] == "loss":
            loss[t0:t1] = torch.where(live, (torch.xlogy(r, r) - r * (z - n[:, None])).sum(1), 0.0)
            lse[t0:t1] = torch.where(live, n, 0.0)
        else:
            g = (torch.exp(z - n[:, None]) - r) * (s["grad_loss"][t0:t1].double().masked_fill(~live, 0.0) / tau)[:, None]
            gh[t0:t1] = g @ W
            gw += g.T @ h
    return {"loss": loss, "lse": lse} if case["call"] == "loss" else {"grad_hidden": gh, "grad_head": gw}


def work(case):
    T, V, d, k = case["rows"], case["vocab"], case["d"], case["top"]
    size = 4 if case["dtype"] == "f32" else 2
    targets = T * (8 * k if k else 4)
    if case["call"] == "loss":
        return {"bytes": (T + V) * d * size + targets + 8 * T, "flops": 2 * T * V * d}
    # the logits again, then both products with their gradient; the log-normalisers and the rows' coefficients are read
    return {"bytes": 2 * (T + V) * d * size + targets + 8 * T, "flops": 6 * T * V * d}
