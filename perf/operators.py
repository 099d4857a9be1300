"""What is measured of the auxiliary losses of a policy's training step.

A case is a plain dict. `kind` says which operator one pass runs, forward and backward:

  distill  distillation from a teacher's top logits over the LM head: per-row loss and log-sum-exp, dH and dW.
           `K` entries a row, `T` the temperature, `rest` whether the teacher's log-sum-exp over its whole vocabulary
           is known (the mass outside the K entries then is one more outcome; without it the K entries are
           renormalised), `top` the type of the teacher's logits, `obs` the share of rows that are masked out
  balance  load-balance loss of a mixture of experts with per-expert counts: loss, counts, sums of probabilities and
           the gradient of the router's logits. `E` experts, `k` of them a token, `score` how logits become
           probabilities, `median` the trajectories' length where each one is balanced by itself (0: the whole batch)

Heads and token counts are those of the repository's configurations (tiny, small, moe, large) and of micro-batches of
them; numbers of experts are generic. Inputs are drawn on the GPU from the seed.
"""
import math

import torch

own = False

DEV = "cuda"

# The heads (hidden size, vocabulary) of the repository's configurations.
HEADS = {"tiny": (256, 4096), "small": (1024, 32000), "moe": (2048, 151936), "large": (6144, 154880)}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _distill(name, head, **kw):
    h, V = HEADS[head]
    return dict(name=name, kind="distill", h=h, V=V, **kw)


def listed():
    return [
        # the tiny configuration in fp32, as in a unit test or a debug run: latency
        _distill("distill_tiny_f32", "tiny", dtype="f32", N=2304, K=8, T=1.0, rest=False, top="f32", obs=0.0),
        # a single token of the moe head: bound by reading W and writing dW
        _distill("distill_one_row", "moe", dtype="bf16", N=1, K=20, T=1.0, rest=True, top="f32", obs=0.0),
        # one short trajectory per micro-batch on the moe head, a server's top 20 log-probs
        _distill("distill_micro", "moe", dtype="bf16", N=517, K=20, T=1.0, rest=True, top="f32", obs=0.25),
        # an fp32 reference run of the small head on one ragged micro-batch
        _distill("distill_small_f32", "small", dtype="f32", N=4099, K=33, T=2.0, rest=True, top="f32", obs=0.25),
        # the small head, many rows, softened and renormalised targets, all rows distilled
        _distill("distill_small_24k", "small", dtype="bf16", N=24576, K=64, T=2.0, rest=False, top="bf16", obs=0.0),
        # the large head on a ragged micro-batch
        _distill("distill_large", "large", dtype="bf16", N=2047, K=50, T=1.0, rest=True, top="f32", obs=0.4),
        # the moe head on the rows of several trajectories, a wide target
        _distill("distill_moe_16k", "moe", dtype="bf16", N=16384, K=128, T=1.0, rest=True, top="bf16", obs=0.25),
        # one short batch through a small router: latency and launches
        dict(name="balance_tiny", kind="balance", dtype="f32", N=2304, E=8, k=2, score="softmax", median=0, obs=0.0),
        # a step of the moe configuration's size, whole batch
        dict(name="balance_64k", kind="balance", dtype="f32", N=65536, E=128, k=8, score="softmax", median=0, obs=0.25),
        # the same tokens, each trajectory balanced by itself, sigmoid scores of a wide router
        dict(name="balance_64k_seq", kind="balance", dtype="bf16", N=65536, E=256, k=8, score="sigmoid", median=4096,
             obs=0.25),
        # rows that are no whole vectors: an odd number of experts
        dict(name="balance_odd", kind="balance", dtype="bf16", N=98301, E=63, k=6, score="softmax", median=1024,
             obs=0.4),
        # a large batch of long trajectories
        dict(name="balance_1m", kind="balance", dtype="bf16", N=(1 << 20) + 333, E=160, k=8, score="softmax", median=0,
             obs=0.25),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n % 2 == 0 and rng.random() < 0.5:  # odd ones among them
        n += 1 if n < hi else -1
    return n


def draw(rng):
    if rng.random() < 0.5:
        c = {"kind": "distill", "dtype": rng.choice(["f32", "bf16", "bf16"])}
        if c["dtype"] == "f32":
            c["h"], c["V"] = rng.choice([96, 256, 515, 1024]), _log_int(rng, 1000, 32000)
            c["N"] = _log_int(rng, 1, 4099)
        else:
            c["h"], c["V"] = HEADS[rng.choice(["tiny", "small", "moe", "large"])]
            if rng.random() < 0.3:
                c["h"], c["V"] = 8 * _log_int(rng, 8, 512), _log_int(rng, 1000, 151936)
            c["N"] = _log_int(rng, 1, min(24576, int(16384.0 * 2048 * 151936 / (c["h"] * c["V"]))))
        c.update(K=_log_int(rng, 1, 256), T=rng.choice([1.0, 1.0, 2.0, 0.7]), rest=rng.random() < 0.5,
                 top=rng.choice(["f32", "bf16"]), obs=rng.choice([0.0, 0.25, 0.4]))
        return c
    c = {"kind": "balance", "dtype": rng.choice(["f32", "bf16"]), "E": _log_int(rng, 4, 512)}
    most = 2.0 * ((1 << 20) + 333) * 160  # logits of the largest listed case, in bytes
    c["N"] = _log_int(rng, 1, int(min(1 << 20, most / (c["E"] * (4 if c["dtype"] == "f32" else 2)))))
    c.update(k=rng.randint(1, min(c["E"], 10)), score=rng.choice(["softmax", "sigmoid"]),
             median=rng.choice([0, 0, _log_int(rng, 64, 8192)]), obs=rng.choice([0.0, 0.25, 0.4]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV, dtype=torch.float32)


def _mask(g, N, obs):
    """Alternating turns: geometric spans of kept rows (mean 256) and of masked ones, `obs` of all rows."""
    if obs == 0.0:
        return None
    mean = 256.0 * obs / (1.0 - obs)
    k = 64 + int(1.6 * N / (256.0 + mean))
    spans = torch.empty(k, 2, device=DEV)
    spans[:, 0].geometric_(1.0 / 256.0, generator=g)
    spans[:, 1].geometric_(1.0 / mean, generator=g)
    kind = torch.tensor([1, 0], dtype=torch.uint8, device=DEV).repeat(k)
    m = torch.repeat_interleave(kind, spans.reshape(-1).long())[:N]
    return torch.cat([m, torch.ones(N - m.numel(), dtype=torch.uint8, device=DEV)])


def _cu(g, N, median):
    """Packed offsets of lognormal (sigma 1) trajectories, `median` tokens or so each and N in all."""
    B = max(1, N // median)
    share = torch.cumsum(torch.empty(B, device=DEV, dtype=torch.float64).log_normal_(0.0, 1.0, generator=g), 0)
    ends = torch.round(share / share[-1] * N)
    return torch.cat([torch.zeros(1, device=DEV, dtype=torch.float64), ends]).to(torch.int32)


def _prepare_distill(case, g, s):
    N, h, V, K = case["N"], case["h"], case["V"], case["K"]
    dt = DTYPES[case["dtype"]]
    s["W"] = (_randn(g, V, h) * 0.02).to(dt)
    # distinct ids a row: two thirds of them among the vocabulary's first (frequent) tokens, the others anywhere after
    # them, each from an arithmetic sequence with a start and a step of the row's own
    often = max(V // 16, K)
    i = torch.arange(K, device=DEV)
    start = torch.randint(0, 1 << 30, (N, 1), generator=g, device=DEV)
    near = torch.randint(0, often // K, (N, 1), generator=g, device=DEV) + 1
    far = torch.randint(0, (V - often) // K, (N, 1), generator=g, device=DEV) + 1
    low, high = (start + i * near) % often, often + (start + i * far) % (V - often)
    ids = torch.where(i % 3 == 2, high, low)
    # a server answers with fewer entries on some rows: the rest of the row is filled with -1
    filled = torch.where(_rand(g, N) < 0.05, (_rand(g, N) * K).long() + 1, K)
    s["ids"] = torch.where(i < filled[:, None], ids, -1).to(torch.int32).contiguous()
    top = 5.0 - 1.3 * torch.log1p(i.float()) + 0.4 * _randn(g, N, K)
    s["top"] = top.to(DTYPES[case["top"]])
    a = torch.where(i < filled[:, None], s["top"].float() / case["T"], -math.inf)
    s["tlse"] = torch.logsumexp(a, 1) - torch.log1p(-(0.02 + 0.3 * _rand(g, N))) if case["rest"] else None
    # a student that has learnt some of it: its logits of the teacher's first three tokens stand out
    H = _randn(g, N, h)
    gain = (math.log(V) + torch.tensor([1.0, 0.0, -1.0], device=DEV) + _randn(g, N, 3)) / (0.0004 * h)
    H += (gain[:, :K, None] * s["W"][s["ids"][:, :3].clamp(min=0).long()].float()).sum(1)
    s["H"] = H.to(dt)
    s["mask"] = _mask(g, N, case["obs"])
    w = (0.5 + _rand(g, N)) / N
    s["grad"] = w if s["mask"] is None else w * s["mask"]


def _prepare_balance(case, g, s):
    N, E, k = case["N"], case["E"], case["k"]
    x = _randn(g, N, E) + 0.7 * _randn(g, E)
    s["logits"] = x.to(DTYPES[case["dtype"]])
    s["experts"] = torch.topk(x, k, dim=1).indices.to(torch.int32).contiguous()
    s["mask"] = _mask(g, N, case["obs"])
    s["cu"] = _cu(g, N, case["median"]) if case["median"] else None
    s["grad"] = torch.full((1,), 0.01, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    (_prepare_distill if case["kind"] == "distill" else _prepare_balance)(case, g, s)
    return s


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------

def _own_distill(s):
    from paper_2607_07508_gb300 import sao
    c = s["case"]
    N, K = s["ids"].shape
    if "ws" not in s:  # what a training program keeps from step to step
        s["ws"] = sao.distill_workspace(N, c["h"], c["V"], K, s["H"].dtype)
        s["loss"], s["lse"], s["lse_rest"] = (torch.empty(N, device=DEV) for _ in range(3))
        s["z_top"] = torch.empty(N, K, device=DEV)
        s["dH"], s["dW"] = torch.empty_like(s["H"]), torch.empty_like(s["W"])
    sao.sao_distill_loss_fwd(s["H"], s["W"], s["ids"], s["top"], c["T"], s["loss"], s["lse"], s["lse_rest"],
                             s["z_top"], s["ws"], teacher_lse=s["tlse"], row_mask=s["mask"])
    sao.sao_distill_loss_bwd(s["H"], s["W"], s["ids"], s["top"], c["T"], s["lse"], s["lse_rest"], s["z_top"],
                             s["grad"], s["dH"], s["dW"], s["ws"], teacher_lse=s["tlse"])
    return {"loss": s["loss"], "lse": s["lse"], "dH": s["dH"], "dW": s["dW"]}


def _own_balance(s):
    from paper_2607_07508_gb300 import sao
    N, E = s["logits"].shape
    B = 1 if s["cu"] is None else s["cu"].numel() - 1
    score = sao.SAO_SCORE_SOFTMAX if s["case"]["score"] == "softmax" else sao.SAO_SCORE_SIGMOID
    if "ws" not in s:
        s["ws"] = sao.balance_workspace(N, E, B)
        s["loss"], s["sums"] = torch.empty(1, device=DEV), torch.empty(B, E, device=DEV)
        s["counts"] = torch.empty(B, E, dtype=torch.int64, device=DEV)
        s["rows"] = torch.empty(B, dtype=torch.int64, device=DEV)
        s["dlogits"] = torch.empty_like(s["logits"])
    sao.sao_balance_loss_fwd(s["logits"], s["experts"], score, s["loss"], s["counts"], s["sums"], s["rows"], s["ws"],
                             row_mask=s["mask"], cu_seqlens=s["cu"])
    sao.sao_balance_loss_bwd(s["logits"], s["experts"].shape[1], score, s["counts"], s["rows"], s["grad"],
                             s["dlogits"], s["ws"], row_mask=s["mask"], cu_seqlens=s["cu"])
    return {"loss": s["loss"], "counts": s["counts"], "sums": s["sums"], "dlogits": s["dlogits"]}


# ---------------------------------------------------------------------------
# their plain form
# ---------------------------------------------------------------------------

def _plain_distill(s):
    c = s["case"]
    T, V = c["T"], c["V"]
    H, W = s["H"].float(), s["W"].float()
    valid = s["ids"] >= 0
    idx = torch.where(valid, s["ids"], V).long()  # entries that say nothing go to a column past the vocabulary
    z = H.new_zeros(H.shape[0], V + 1)
    z[:, :V] = (H @ W.T) / T
    zt = z.gather(1, idx)
    z[:, V] = -math.inf
    z.scatter_(1, idx, -math.inf)  # from here on: the logits outside the teacher's entries
    top = torch.where(valid, zt, -math.inf)
    m_rest, m_top = z.amax(1), top.amax(1)
    m = torch.maximum(m_rest, m_top)
    e_rest, e_top = torch.exp(z - m_rest[:, None]), torch.exp(top - m[:, None])
    sum_rest = e_rest.sum(1)
    lse_rest = m_rest + torch.log(sum_rest)
    lse = m + torch.log(torch.exp(lse_rest - m) + e_top.sum(1))
    a = torch.where(valid, s["top"].float() / T, -math.inf)
    if s["tlse"] is None:
        m_a = a.amax(1)
        la = m_a + torch.log(torch.exp(a - m_a[:, None]).sum(1))
        p = torch.exp(a - la[:, None])
        rho = torch.zeros_like(la)
    else:
        la = s["tlse"]
        p = torch.exp(a - la[:, None])
        rho = (1.0 - p.sum(1)).clamp(min=0.0)
    log_q_rest = lse_rest - lse
    terms = torch.where(p > 0, p * (a - la[:, None] - zt + lse[:, None]), 0.0)
    loss = terms.sum(1) + torch.where(rho > 0, rho * (torch.log(rho) - log_q_rest), 0.0)
    if s["mask"] is not None:
        keep = s["mask"] != 0
        loss, lse = torch.where(keep, loss, 0.0), torch.where(keep, lse, 0.0)
    scale = s["grad"] / T
    dz = e_rest * ((torch.exp(log_q_rest) - rho) / sum_rest * scale)[:, None]
    q_top = torch.exp(top - (m_rest + torch.log(sum_rest) - log_q_rest)[:, None])
    dz.scatter_(1, idx, (q_top - p) * scale[:, None])
    dz = dz[:, :V]
    return {"loss": loss, "lse": lse, "dH": (dz @ W).to(s["H"].dtype), "dW": (dz.T @ H).to(s["W"].dtype)}


def _plain_balance(s):
    c = s["case"]
    x = s["logits"].float()
    N, E = x.shape
    k = s["experts"].shape[1]
    keep = torch.ones(N, device=DEV) if s["mask"] is None else s["mask"].float()
    if c["score"] == "softmax":
        e = torch.exp(x - x.amax(1, keepdim=True))
        prob = e / e.sum(1, keepdim=True)
        slope = prob
    else:
        e = 1.0 / (1.0 + torch.exp(-x))
        prob = e / e.sum(1, keepdim=True)
        slope = prob / (1.0 + torch.exp(x))
    kept = prob * keep[:, None]
    if s["cu"] is None:
        B = 1
        seg = torch.zeros(N, dtype=torch.int64, device=DEV)
        rows, sums = keep.sum().reshape(1), kept.sum(0, keepdim=True)
    else:
        B = s["cu"].numel() - 1
        seg = torch.bucketize(torch.arange(N, device=DEV, dtype=torch.int32), s["cu"][1:], right=True)
        rows = torch.zeros(B, device=DEV).index_add_(0, seg, keep)
        sums = torch.zeros(B, E, device=DEV).index_add_(0, seg, kept)
    slot = (seg[:, None] * E + s["experts"]).reshape(-1)
    counts = torch.zeros(B * E, dtype=torch.int64, device=DEV).index_add_(
        0, slot, keep.long().repeat_interleave(k)).reshape(B, E)
    used = (rows > 0).sum().clamp(min=1)
    w = counts.float() * (E / (k * rows.clamp(min=1).square() * used))[:, None]
    loss = (w * sums).sum().reshape(1)
    w = w * s["grad"]
    wt = w[seg]
    d = slope * (wt - (prob * wt).sum(1, keepdim=True)) * keep[:, None]
    return {"loss": loss, "counts": counts, "sums": sums, "dlogits": d.to(s["logits"].dtype)}


def run(s):
    if s["case"]["kind"] == "distill":
        return _own_distill(s) if own else _plain_distill(s)
    return _own_balance(s) if own else _plain_balance(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------

def work(case):
    N = case["N"]
    size = 2 if case["dtype"] == "bf16" else 4
    rows = N * (1.0 - case["obs"])
    if case["kind"] == "distill":
        h, V, K = case["h"], case["V"], case["K"]
        top = 2 if case["top"] == "bf16" else 4
        return {"bytes": 2.0 * size * (N * h + V * h) + rows * K * (4 + top) + 12.0 * N, "flops": 6.0 * rows * h * V}
    return {"bytes": size * case["E"] * (rows + N) + rows * case["k"] * 4, "flops": 20.0 * rows * case["E"]}


def exact(case, seed):
    """From the losses' definitions in 64 bits, their gradients by differentiating them."""
    s = prepare(case, seed)
    N = case["N"]
    keep = torch.ones(N, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    if case["kind"] == "balance":
        x = s["logits"].double().requires_grad_()
        score = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
        score = score / score.sum(1, keepdim=True)
        cu = [0, N] if s["cu"] is None else s["cu"].tolist()
        E, k = case["E"], case["k"]
        counts, sums, terms = [], [], []
        for b, e in zip(cu[:-1], cu[1:]):
            on = keep[b:e]
            n = int(on.sum())
            counts.append(torch.bincount(s["experts"][b:e][on].reshape(-1).long(), minlength=E))
            sums.append(score[b:e][on].sum(0))
            if n:
                terms.append((counts[-1] * (E / (k * n)) * sums[-1] / n).sum())
        loss = sum(terms) / len(terms) if terms else x.sum() * 0.0
        grad, = torch.autograd.grad(loss * s["grad"].double()[0], x)
        return {"loss": loss.detach().reshape(1), "counts": None, "sums": torch.stack(sums).detach(), "dlogits": grad}
    if 6.0 * N * case["h"] * case["V"] > 1.3e13:
        return None
    T, V = case["T"], case["V"]
    W = s["W"].double()
    dW = torch.zeros_like(W)
    dH = torch.zeros(N, case["h"], dtype=torch.float64, device=DEV)
    loss, lse = torch.zeros(N, dtype=torch.float64, device=DEV), torch.zeros(N, dtype=torch.float64, device=DEV)
    rows = keep.nonzero()[:, 0]
    for at in range(0, rows.numel(), 2048):
        t = rows[at:at + 2048]
        H = s["H"][t].double()
        z = (H @ W.T / T).requires_grad_()
        ids, a = s["ids"][t].long(), s["top"][t].double() / T
        valid = ids >= 0
        total = torch.logsumexp(z, 1)
        inside = torch.zeros(t.numel(), V + 1, dtype=torch.bool, device=DEV)
        inside.scatter_(1, torch.where(valid, ids, V), True)
        log_q = torch.log_softmax(z, 1).gather(1, ids.clamp(min=0))
        whole = torch.logsumexp(a.masked_fill(~valid, -math.inf), 1) if s["tlse"] is None else s["tlse"][t].double()
        log_p = a - whole[:, None]
        kl = (torch.exp(log_p) * (log_p - log_q)).masked_fill(~valid, 0.0).sum(1)
        if s["tlse"] is not None:
            left = 1.0 - torch.exp(log_p).masked_fill(~valid, 0.0).sum(1)
            rest = torch.logsumexp(z.masked_fill(inside[:, :V], -math.inf), 1) - total
            kl = kl + left * (torch.log(left) - rest)
        dz, = torch.autograd.grad((kl * s["grad"][t].double()).sum(), z)
        loss[t], lse[t] = kl.detach(), total.detach()
        dH[t] = dz @ W / T
        dW += dz.T @ H / T
    return {"loss": loss, "lse": lse, "dH": dH, "dW": dW}
