"""The operators around the loss head in one step, as the example chains them: each against its plain form in 64 bits on
what it was given, and the calls captured together.

Bounds with u = 2^-24 and a bf16 rounding of 2^-8 of a value: weights 80 u (sigmoids of logits up to 10); the stream one
rounding of its sum, H 34 u and one; the norm's gradients 64 u of their terms and one rounding; the router's 80 u of its
terms and two roundings (its own sum with the balance loss's, once more each); the global norm 6 u, and clipped gradients
7 u and one rounding."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao
from tests import _route as R

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8


def test_whole_step():
    from examples import moe_policy_step as M
    b = M.batch()
    l = M.layer(b)
    o = M.whole_step(b, l)
    torch.cuda.synchronize()
    x = b["router"]
    on = torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
    assert torch.equal(o["experts"], R.choose(x, M.CHOSEN, "sigmoid", l["bias"], 4, 2, True))
    w = R.weights(x, o["experts"], "sigmoid", True, M.ROUTE_SCALE, on)
    assert ((o["weights"].double() - w).abs() <= 80 * U * w).all()

    total = o["answer"].double() + l["residual"].double()
    assert ((o["stream"].double() - total).abs() <= (U + HALF) * total.abs()).all()
    r, g = o["stream"].double(), l["norm_weight"].double()
    rstd = (r.pow(2).mean(1, keepdim=True) + M.EPS).rsqrt()
    H = r * rstd * g
    assert ((o["H"].double() - H).abs() <= (34 * U + HALF) * H.abs()).all()

    dy = o["dH_rounded"].double()
    a = dy * g
    d = rstd * a - r * (a * r).mean(1, keepdim=True) * rstd ** 3
    size = rstd * a.abs() + r.abs() * (a * r).abs().mean(1, keepdim=True) * rstd ** 3
    assert ((o["d_stream"].double() - d).abs() <= 64 * U * size + HALF * d.abs()).all()
    terms = dy * r * rstd
    assert ((o["d_norm"].double() - terms.sum(0)).abs() <= 66 * U * terms.abs().sum(0)).all()

    d, size = R.gradient(x, o["experts"], w, o["d_weights"], "sigmoid", True, M.ROUTE_SCALE, on)
    d = d + o["balance_router"].double()
    assert ((o["d_router"].double() - d).abs() <= 80 * U * size + (HALF + U) * d.abs()).all()

    grads = [o["dW"], o["d_norm"], o["d_router"]]
    norm = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in grads))
    assert abs(o["norm"].item() - norm) <= 6 * U * norm and norm > M.MAX_NORM
    for t, c in zip(grads, o["clipped"]):
        want = t.double() * (M.MAX_NORM / norm)
        assert ((c.double() - want).abs() <= (7 * U + torch.finfo(t.dtype).eps / 2) * want.abs() + 2.0 ** -134).all()


def _chain(s):
    """Route, norm, their gradients and the clipping, with one workspace for all."""
    sao.sao_route_fwd(s["x"], 0, s["ids"], s["w"], s["ws"], bias=s["bias"])
    sao.sao_rms_norm_fwd(s["h"], s["g"], 1e-6, s["ws"], residual=s["res"], sum=s["sum"], y=s["y"], rstd=s["rstd"])
    sao.sao_rms_norm_bwd(s["sum"], s["g"], s["rstd"], s["y"], s["dh"], s["dg"], s["ws"])
    sao.sao_route_bwd(s["x"], 0, s["ids"], s["w"], s["w"], s["dx"], s["ws"])
    sao.sao_grad_sumsq(s["grads"], s["sumsq"], s["ws"])
    sao.sao_grad_clip(s["grads"], s["sumsq"], 0.1, s["norm"], s["coef"], s["ws"])


def _state(N, E, k, h, ws, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    s = {"x": r(N, E).cuda(), "bias": (0.1 * r(E)).cuda(), "h": r(N, h).bfloat16().cuda(), "res": r(N, h).bfloat16().cuda(),
         "g": r(h).cuda(), "ids": torch.zeros(N, k, dtype=torch.int32, device="cuda"), "w": torch.zeros(N, k, device="cuda"),
         "rstd": torch.zeros(N, device="cuda"), "dg": torch.zeros(h, device="cuda"), "ws": ws,
         "sumsq": torch.zeros(1, dtype=torch.float64, device="cuda"), "norm": torch.zeros(1, device="cuda"),
         "coef": torch.zeros(1, device="cuda")}
    s.update({n: torch.zeros_like(s["h"]) for n in ("sum", "y", "dh")}, dx=torch.zeros_like(s["x"]))
    s["grads"] = sao.TensorList([s["dx"], s["dg"], s["dh"]])
    return s


OUT = ("ids", "w", "sum", "y", "rstd", "dh", "dg", "dx", "sumsq", "norm", "coef")


def test_graphs_share_a_workspace():
    """Two captured chains of different sizes over one workspace, replayed in turn, give what eager calls give."""
    ws = torch.empty(max(sao.sao_norm_workspace_bytes(4000, 520), sao.sao_route_workspace_bytes(4000, 64),
                         sao.sao_grad_workspace_bytes()), dtype=torch.uint8, device="cuda")
    states = [_state(4000, 64, 8, 520, ws, 1), _state(33, 17, 3, 96, ws, 2)]
    want = []
    for s in states:
        _chain(s)
        torch.cuda.synchronize()
        want.append([s[k].clone() for k in OUT])
    graphs = []
    for s in states:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            _chain(s)
    for _ in range(3):
        for s in states:
            for k in OUT:
                s[k].zero_()
        ws.fill_(255)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(states, want):
            assert all(torch.equal(s[k], v) for k, v in zip(OUT, w))


def test_two_streams_with_a_workspace_each():
    """Chains on two streams at once, many times, with inputs that differ."""
    size = max(sao.sao_norm_workspace_bytes(4000, 520), sao.sao_grad_workspace_bytes())
    states = [_state(4000, 64, 8, 520, torch.empty(size, dtype=torch.uint8, device="cuda"), s) for s in (3, 4)]
    want = []
    for s in states:
        _chain(s)
        torch.cuda.synchronize()
        want.append([s[k].clone() for k in OUT])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, stream in zip(states, streams):
            with torch.cuda.stream(stream):
                _chain(s)
    torch.cuda.synchronize()
    for s, w in zip(states, want):
        assert all(torch.equal(s[k], v) for k, v in zip(OUT, w))


def test_checked_mode():
    """The calls between a device check before and after them: nothing to report, and what they give stays the same."""
    ws = torch.empty(sao.sao_norm_workspace_bytes(4000, 520), dtype=torch.uint8, device="cuda")
    s = _state(300, 64, 8, 96, ws, 5)
    _chain(s)
    torch.cuda.synchronize()
    want = [s[k].clone() for k in OUT]
    sao.sao_set_checked(True)
    try:
        _chain(s)
    finally:
        sao.sao_set_checked(False)
    assert all(torch.equal(s[k], v) for k, v in zip(OUT, want))
