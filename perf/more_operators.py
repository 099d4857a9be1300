"""What is measured of the operators around the loss head of a policy's training step.

A case is a plain dict. `kind` says which operator one pass runs:

  route  routing to experts: choices and weights (forward), with `train` the gradient of the router's logits too. `E`
         experts, `k` a token, `score` softmax or sigmoid, `bias` whether a balance bias takes part in the choice,
         `groups` of experts of which `kept` stay (1, 1: no groups) by their best expert or the sum of their best `two`,
         `renorm` whether a token's weights add up to the factor, `replay` whether the rollout's choices are given,
         `obs` the share of rows that are masked out
  norm   root-mean-square norm of the sum of a layer's output and the residual stream: the new stream and the normed
         rows, in 8 bits with scales for `scaling` row, block (128 columns) or mx (32 columns, powers of two); with `train`
         the gradients of the stream and the weight too
  clip   the global norm of all gradients and their clipped copies: the head's fp32 gradient (`head` rows), `layers`
         layers of bf16 ones of hidden size h, fp32 gradients of the norms' weights

Hidden sizes, vocabularies and token counts are those of the repository's configurations and of micro-batches of them;
numbers of experts and layers are generic. Inputs are drawn on the GPU from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOWEST_SCALE = 2.0 ** -126
BLOCK = {"block": 128, "mx": 32}


def _route(name, N, E, k, dtype, score, bias=False, groups=1, kept=1, two=False, renorm=True, replay=False, obs=0.0,
           train=True):
    return dict(name=name, kind="route", N=N, E=E, k=k, dtype=dtype, score=score, bias=bias, groups=groups, kept=kept,
                two=two, renorm=renorm, replay=replay, obs=obs, train=train)


def _norm(name, N, h, dtype, residual=True, scaling="none", train=True):
    return dict(name=name, kind="norm", N=N, h=h, dtype=dtype, residual=residual, scaling=scaling, train=train)


def _clip(name, head, h, layers, limit):
    return dict(name=name, kind="clip", head=head, h=h, layers=layers, limit=limit)


def listed():
    return [
        # a decode step of a rollout: a few tokens through a wide grouped router, forward alone
        _route("route_decode", 7, 256, 8, "f32", "sigmoid", bias=True, groups=8, kept=4, two=True, train=False),
        # a step of the moe configuration's size
        _route("route_64k", 65536, 128, 8, "f32", "softmax"),
        # the same tokens through a wide grouped router with a balance bias, prompts and observations masked out
        _route("route_64k_groups", 65536, 256, 8, "bf16", "sigmoid", bias=True, groups=8, kept=4, two=True, obs=0.25),
        # rows that are no whole vectors, weights that are the probabilities: a gradient of every logit
        _route("route_odd", 98301, 63, 6, "bf16", "softmax", renorm=False),
        # a large batch of long trajectories
        _route("route_1m", (1 << 20) + 333, 160, 8, "bf16", "softmax", groups=8, kept=3),
        # a decode step of the moe configuration, normed rows in 8 bits for the rollout's products
        _norm("norm_decode", 3, 2048, "bf16", scaling="block", train=False),
        # an fp32 reference run of an odd hidden size, a ragged micro-batch
        _norm("norm_odd_f32", 4099, 515, "f32"),
        # a prefill's rows of the large configuration, in 8 bits with a power of two for each 32
        _norm("norm_large_mx", 16384, 6144, "bf16", scaling="mx", train=False),
        # a step of the moe configuration's size
        _norm("norm_64k", 65536, 2048, "bf16"),
        # the tiny configuration: a few small tensors, latency
        _clip("clip_tiny", 4096, 256, 2, 0.5),
        # the small configuration's head and a few layers: what the L2 holds
        _clip("clip_small", 32000, 1024, 8, 1.0),
        # the moe configuration's head and the dense part of its layers
        _clip("clip_moe", 151936, 2048, 48, 1.0),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n % 2 == 0 and rng.random() < 0.5:  # odd ones among them
        n += 1 if n < hi else -1
    return n


def draw(rng):
    kind = rng.choice(["route", "norm", "clip"])
    if kind == "route":
        c = {"kind": "route", "dtype": rng.choice(["f32", "bf16"]), "E": _log_int(rng, 4, 512), "groups": 1, "kept": 1}
        if rng.random() < 0.5:
            c["groups"] = rng.choice([2, 4, 5, 8, 16])
            c["E"] = c["groups"] * max(1, c["E"] // c["groups"])
            c["kept"] = rng.randint(1, c["groups"])
        most = 2.0 * ((1 << 20) + 333) * 160  # bytes of logits of the largest listed case
        c["N"] = _log_int(rng, 1, int(min(1 << 20, most / (c["E"] * (4 if c["dtype"] == "f32" else 2)))))
        c["k"] = rng.randint(1, min(10, c["E"] // c["groups"] * c["kept"]))
        c.update(score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, two=rng.random() < 0.5,
                 renorm=c["k"] > 1 and rng.random() < 0.6, replay=rng.random() < 0.15, obs=rng.choice([0.0, 0.25, 0.4]),
                 train=rng.random() < 0.7)
        return c
    if kind == "norm":
        c = {"kind": "norm", "dtype": rng.choice(["f32", "bf16", "bf16"]), "h": rng.choice([256, 1024, 2048, 4096, 6144])}
        if rng.random() < 0.5:
            c["h"] = _log_int(rng, 8, 8192)
        most = 2.0 * 65536 * 2048  # bytes of an array of the largest listed case
        c["N"] = _log_int(rng, 1, int(min(1 << 20, most / (c["h"] * (4 if c["dtype"] == "f32" else 2)))))
        c.update(residual=rng.random() < 0.8, train=rng.random() < 0.6)
        c["scaling"] = "none" if c["train"] else rng.choice(["none", "row", "block", "mx"])
        return c
    h = rng.choice([256, 1024, 2048]) if rng.random() < 0.6 else _log_int(rng, 16, 2048)
    return {"kind": "clip", "head": _log_int(rng, 16, 151936), "h": h, "layers": rng.randint(0, 48),
            "limit": rng.choice([0.1, 1.0, 1.0, 1e6])}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


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


def _prepare_route(case, g, s):
    N, E, k = case["N"], case["E"], case["k"]
    x = _randn(g, N, E) + 0.7 * _randn(g, E)
    s["logits"] = x.to(DTYPES[case["dtype"]])
    s["bias"] = 0.1 * _randn(g, E) if case["bias"] else None
    s["mask"] = _mask(g, N, case["obs"])
    s["grad"] = _randn(g, N, k) / N
    # a rollout's choices: by logits that moved a little since
    s["given"] = (torch.topk(x + 0.05 * _randn(g, N, E), k, dim=1).indices.to(torch.int32).contiguous()
                  if case["replay"] else None)


def _prepare_norm(case, g, s):
    N, h, dt = case["N"], case["h"], DTYPES[case["dtype"]]
    s["x"] = (0.5 * _randn(g, N, h)).to(dt)
    # a residual stream has a few columns that are much larger than the others
    s["residual"] = (_randn(g, N, h) * (1.0 + 8.0 * (_randn(g, h) > 2.5))).to(dt) if case["residual"] else None
    s["weight"] = 1.0 + 0.2 * _randn(g, h)
    if case["train"]:
        s["dy"], s["dsum"] = (_randn(g, N, h) / N).to(dt), (_randn(g, N, h) / N).to(dt)


def _clip_shapes(case):
    """(elements, type) of the gradients: the head, the last norm, the layers' products and norms."""
    h, layers = case["h"], case["layers"]
    return ([(case["head"] * h, torch.float32), (h, torch.float32)] +
            [(h * h, torch.bfloat16), (h * h // 2, torch.bfloat16), (h, torch.float32)] * layers)


def _prepare_clip(case, g, s):
    shapes = _clip_shapes(case)
    total = sum(n for n, _ in shapes)
    s["grads"] = [(_randn(g, n) * (2.0 / math.sqrt(total))).to(dt) for n, dt in shapes]
    # the clipped copies lie in one flat buffer of each type, as an optimiser keeps them, every one on 16 bytes
    at, places = {torch.float32: 0, torch.bfloat16: 0}, []
    for n, dt in shapes:
        places.append((dt, at[dt], n))
        at[dt] += -(-n // 8) * 8
    s["flat"] = {dt: torch.zeros(n, dtype=dt, device=DEV) for dt, n in at.items()}
    s["out"] = [s["flat"][dt][i:i + n] for dt, i, n in places]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    {"route": _prepare_route, "norm": _prepare_norm, "clip": _prepare_clip}[case["kind"]](case, g, s)
    return s


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------

def _own_route(s):
    from paper_2607_07508_gb300 import sao
    c = s["case"]
    N, E = s["logits"].shape
    k = c["k"]
    score = sao.SAO_SCORE_SOFTMAX if c["score"] == "softmax" else sao.SAO_SCORE_SIGMOID
    if "ws" not in s:  # what a training program keeps from step to step
        s["ws"] = sao.route_workspace(N, E)
        s["ids"] = s["given"] if c["replay"] else torch.empty(N, k, dtype=torch.int32, device=DEV)
        s["weights"] = torch.empty(N, k, device=DEV)
        s["dlogits"] = torch.empty_like(s["logits"])
    sao.sao_route_fwd(s["logits"], score, s["ids"], s["weights"], s["ws"], bias=s["bias"], row_mask=s["mask"],
                      groups=c["groups"], groups_kept=c["kept"],
                      group_score=sao.SAO_GROUP_TOP2 if c["two"] else sao.SAO_GROUP_MAX, renormalise=c["renorm"],
                      scale=2.5, replay=c["replay"])
    out = {"ids": s["ids"], "weights": s["weights"]}
    if c["train"]:
        sao.sao_route_bwd(s["logits"], score, s["ids"], s["weights"], s["grad"], s["dlogits"], s["ws"],
                          row_mask=s["mask"], renormalise=c["renorm"], scale=2.5)
        out["dlogits"] = s["dlogits"]
    return out


def _own_norm(s):
    from paper_2607_07508_gb300 import sao
    c = s["case"]
    x, h = s["x"], c["h"]
    N = x.shape[0]
    if "ws" not in s:
        s["ws"] = sao.norm_workspace(N, h)
        s["sum"] = torch.empty_like(x) if c["residual"] else None
        s["rstd"] = torch.empty(N, device=DEV) if c["train"] else None
        s["y"] = torch.empty_like(x) if c["scaling"] == "none" else None
        s["y8"], s["scales"] = sao.norm_out8(N, h, c["scaling"], device=DEV) if c["scaling"] != "none" else (None, None)
        if c["train"]:
            s["dx"], s["dw"] = torch.empty_like(x), torch.empty(h, device=DEV)
    sao.sao_rms_norm_fwd(x, s["weight"], 1e-6, s["ws"], residual=s["residual"], sum=s["sum"], y=s["y"], rstd=s["rstd"],
                         y8=s["y8"], scales=s["scales"], scaling=c["scaling"])
    out = {"sum": s["sum"], "y": s["y"]}
    if c["train"]:
        sao.sao_rms_norm_bwd(s["sum"] if c["residual"] else x, s["weight"], s["rstd"], s["dy"], s["dx"], s["dw"],
                             s["ws"], dsum=s["dsum"])
        out.update(rstd=s["rstd"], dx=s["dx"], dw=s["dw"])
    if c["scaling"] != "none":
        out.update(y8=s["y8"], scales=s["scales"])
    return out


def _own_clip(s):
    from paper_2607_07508_gb300 import sao
    if "ws" not in s:
        s["ws"] = sao.grad_workspace()
        s["sumsq"] = torch.empty(1, dtype=torch.float64, device=DEV)
        s["norm"], s["coef"] = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
        s["list"], s["out_list"] = sao.TensorList(s["grads"]), sao.TensorList(s["out"])
    sao.sao_grad_sumsq(s["list"], s["sumsq"], s["ws"])
    sao.sao_grad_clip(s["list"], s["sumsq"], s["case"]["limit"], s["norm"], s["coef"], s["ws"], out=s["out_list"])
    return {"norm": s["norm"], "coef": s["coef"], "f32": s["flat"][torch.float32], "bf16": s["flat"][torch.bfloat16]}


# ---------------------------------------------------------------------------
# their plain form
# ---------------------------------------------------------------------------

def _plain_route(s):
    c = s["case"]
    x = s["logits"].double()  # in 64 bits: experts next to one another at the border of the choice
    N, E = x.shape
    k, G = c["k"], c["groups"]
    keep = torch.ones(N, 1, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"][:, None] != 0
    if c["score"] == "softmax":
        e = torch.exp(x - x.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    if c["replay"]:
        ids = s["given"].long()
    else:
        key = score if s["bias"] is None else score + s["bias"].double()
        if G > 1:
            by_group = torch.sort(key.reshape(N, G, E // G), dim=2, descending=True).values
            value = by_group[:, :, :2].sum(2) if c["two"] else by_group[:, :, 0]
            best = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :c["kept"]]
            stays = torch.zeros(N, G, dtype=torch.bool, device=DEV).scatter_(1, best, True)
            key = torch.where(stays[:, :, None], key.reshape(N, G, E // G), -math.inf).reshape(N, E)
        ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k]
    w = score.gather(1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    w = torch.where(keep, 2.5 * w, 0.0).float()
    out = {"ids": s["given"] if c["replay"] else torch.where(keep, ids, -1).to(torch.int32), "weights": w}
    if c["train"]:
        g, score = s["grad"], score.float()
        mean = (g * w).sum(1, keepdim=True)
        if c["score"] == "sigmoid":  # 1 - sigmoid(x) as sigmoid(-x)
            slope = 1.0 / (1.0 + torch.exp(s["logits"].float().gather(1, ids)))
        else:
            slope = 1.0
        d = torch.zeros(N, E, device=DEV)
        if c["renorm"]:
            d.scatter_(1, ids, slope * w * (g - mean / 2.5))
        elif c["score"] == "sigmoid":
            d.scatter_(1, ids, slope * w * g)
        else:
            d.scatter_(1, ids, 2.5 * g)
            d = score * (d - mean)
        out["dlogits"] = torch.where(keep, d, 0.0).to(s["logits"].dtype)
    return out


def _plain_norm(s):
    c = s["case"]
    x, h = s["x"], c["h"]
    N = x.shape[0]
    r = x.float()
    out = {"sum": None, "y": None}
    if c["residual"]:
        out["sum"] = (r + s["residual"].float()).to(x.dtype)
        r = out["sum"].float()
    rstd = 1.0 / torch.sqrt((r * r).sum(1, keepdim=True) / h + 1e-6)
    y = r * rstd * s["weight"]
    if c["scaling"] == "none":
        out["y"] = y.to(x.dtype)
    else:
        size = BLOCK.get(c["scaling"], h)
        blocks = torch.nn.functional.pad(y, (0, -h % size)).reshape(N, -1, size)
        scale = blocks.abs().amax(2, keepdim=True) / 448.0
        if c["scaling"] == "mx":
            f, e = torch.frexp(scale)
            e = torch.where(f == 0.5, e - 1, e).clamp(-127, 127)
            scale = torch.exp2(torch.where(scale > 0, e, -127).double()).float()
        else:
            scale = scale.clamp(min=LOWEST_SCALE)
        out["y8"] = (blocks / scale).reshape(N, -1)[:, :h].to(torch.float8_e4m3fn)
        out["scales"] = scale[:, :, 0].to(torch.float8_e8m0fnu if c["scaling"] == "mx" else torch.float32)
    if c["train"]:
        dy = s["dy"].float()
        a, xhat = dy * s["weight"], r * rstd
        d = rstd * (a - xhat * ((a * xhat).sum(1, keepdim=True) / h)) + s["dsum"].float()
        out.update(rstd=rstd[:, 0], dx=d.to(x.dtype), dw=(dy * xhat).sum(0))
    return out


def _plain_clip(s):
    # in 64 bits: a sum of up to half a billion squares
    flat = torch.cat([g.float() for g in s["grads"]])
    norm = torch.sqrt((flat.double() ** 2).sum().reshape(1))
    limit = s["case"]["limit"]
    coef = torch.where(norm > limit, limit / norm, 1.0).float()
    parts = torch.split(flat * coef, [g.numel() for g in s["grads"]])
    for out, part in zip(s["out"], parts):
        out.copy_(part)
    return {"norm": norm.float(), "coef": coef, "f32": s["flat"][torch.float32], "bf16": s["flat"][torch.bfloat16]}


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"route": _own_route, "norm": _own_norm, "clip": _own_clip}[kind](s)
    return {"route": _plain_route, "norm": _plain_norm, "clip": _plain_clip}[kind](s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------

def work(case):
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "route":
        N, E, k = case["N"], case["E"], case["k"]
        rows = N * (1.0 - case["obs"])
        logits = rows * (k if case["replay"] and case["renorm"] else E) * size
        return {"bytes": logits + 8.0 * N * k + ((N * E * size + 4.0 * rows * k) if case["train"] else 0.0),
                "flops": 20.0 * rows * E}
    if case["kind"] == "norm":
        N, h = case["N"], case["h"]
        read = 2 if case["residual"] else 1
        out = size if case["scaling"] == "none" else 1.0 + {"row": 0.0, "block": 4.0 / 128, "mx": 1.0 / 32}[case["scaling"]]
        return {"bytes": N * h * (size * (2 * read - 1) + out + (3 * size if case["train"] else 0)) + 4.0 * h,
                "flops": N * h * (16.0 if case["train"] else 6.0)}
    shapes = _clip_shapes(case)
    return {"bytes": 2.0 * sum(n * (4 if dt == torch.float32 else 2) for n, dt in shapes),
            "flops": 3.0 * sum(n for n, _ in shapes)}


def _chosen(x, score, case, bias):
    """The choices from their definition: one group, one expert at a time, the first of the best."""
    N, E = x.shape
    key = score.detach().clone()
    if bias is not None:
        key += bias.double()
    G, rows = case["groups"], torch.arange(N, device=DEV)
    if G > 1:
        top = key.reshape(N, G, E // G).topk(min(2, E // G), dim=2).values
        value = top.sum(2) if case["two"] else top[:, :, 0].clone()
        out = torch.ones(N, G, dtype=torch.bool, device=DEV)
        for _ in range(case["kept"]):
            best = value.argmax(1)
            out[rows, best], value[rows, best] = False, -math.inf
        key = key.masked_fill(out.repeat_interleave(E // G, 1), -math.inf)
    ids = []
    for _ in range(case["k"]):
        ids.append(key.argmax(1))
        key[rows, ids[-1]] = -math.inf
    return torch.stack(ids, 1)


def _exact_route(case, s):
    x = s["logits"].double().requires_grad_()
    on = torch.ones(case["N"], device=DEV) if s["mask"] is None else s["mask"].float()
    score = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
    ids = s["given"].long() if case["replay"] else _chosen(x, score, case, s["bias"])
    w = score.gather(1, ids)
    if case["renorm"]:  # as logarithms: sums of scores that are all small
        log = torch.log_softmax(x, 1) if case["score"] == "softmax" else torch.nn.functional.logsigmoid(x)
        w = torch.softmax(log.gather(1, ids), 1)
    w = 2.5 * w * on[:, None]
    out = {"ids": None, "weights": w.detach()}
    if case["train"]:
        out["dlogits"], = torch.autograd.grad((w * s["grad"].double()).sum(), x)
    return out


def _exact_norm(case, s):
    x = s["x"].double()
    out = {"sum": None, "y": None}
    if case["residual"]:
        out["sum"] = x + s["residual"].double()
        x = out["sum"].to(s["x"].dtype).double()  # the norm is that of the stream as it is stored
    r, w = x.requires_grad_(), s["weight"].double().requires_grad_()
    rstd = (r.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt()
    y = r * rstd * w
    if case["scaling"] == "none":
        out["y"] = y.detach()
    else:
        out.update(y8=None, scales=None)
        if case["scaling"] != "mx":
            size = BLOCK.get(case["scaling"], case["h"])
            out["scales"] = torch.stack([b.abs().amax(1) for b in y.detach().split(size, 1)], 1) / 448.0
    if case["train"]:
        dx, dw = torch.autograd.grad((y * s["dy"].double()).sum(), (r, w))
        out.update(rstd=rstd.detach()[:, 0], dx=dx + s["dsum"].double(), dw=dw)
    return out


def _exact_clip(case, s):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
    coef = min(1.0, case["limit"] / norm)
    for g, out in zip(s["grads"], s["out"]):
        out.copy_(torch.full_like(g, 1.0))
    flat = {dt: t.double() for dt, t in s["flat"].items()}
    for dt, t in flat.items():
        t[t != 0] = torch.cat([g.double() for g in s["grads"] if g.dtype is dt] or [t[:0]])
        t *= coef
    one = lambda v: torch.full((1,), v, dtype=torch.float64, device=DEV)  # noqa: E731
    return {"norm": one(norm), "coef": one(coef), "f32": flat[torch.float32], "bf16": flat[torch.bfloat16]}


def exact(case, seed):
    """From the operators' definitions in 64 bits, gradients by differentiating them."""
    s = prepare(case, seed)
    return {"route": _exact_route, "norm": _exact_norm, "clip": _exact_clip}[case["kind"]](case, s)
