"""Root-mean-square norm against fp64.

Bounds with u = 2^-24, at worst: a mean of squares is a chain of 32 in a lane, 5 halvings and 16 warps, and the squares'
rounding: 54 u, half of it behind the root; with the quotient, the mean's factor and eps rstd is off by 32 u. y has two
more roundings and its own; an 8-bit value (of v = y / scale, with scale's own two roundings, 40 u) half a step, 2^-4 of itself or
2^-10 among the denormal ones. dx: 64 u of the largest of each of its terms, and its rounding. dw: a chain of rows, of
teams, of parts and the rounding of its terms, 64 u of the sum of their absolute values up to 5,000 rows."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def half(t):
    return torch.finfo(t.dtype).eps / 2


def _place(t, offset):
    """t on the GPU, `offset` elements behind 16 bytes."""
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    return flat[offset:].view(t.shape).copy_(t)


def _case(N, h, dtype="bf16", w_dtype="f32", residual=True, seed=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    c = {"x": r(N, h), "dy": r(N, h) / N, "dsum": r(N, h) / N, "residual": r(N, h) * (1 + 8 * (r(h) > 2)) if residual else None}
    c = {k: None if v is None else _place(v.to(DT[dtype]), offset) for k, v in c.items()}
    c["weight"] = _place((1 + 0.3 * r(h)).to(DT[w_dtype]), offset)
    return c


def _new(like, offset=0):
    return _place(torch.full(like.shape, math.nan, dtype=like.dtype), offset)


def forward(c, eps=1e-6, scaling="none", want_y=True, rstd=True, offset=0, stream=None):
    x, res = c["x"], c["residual"]
    N, h = x.shape
    o = {"sum": None if res is None else _new(x, offset), "y": _new(x, offset) if want_y else None,
         "rstd": torch.full((N,), math.nan, device="cuda") if rstd else None, "y8": None, "scales": None}
    if scaling != "none":
        o["y8"], o["scales"] = sao.norm_out8(N, h, scaling)
        o["y8"].view(torch.uint8).fill_(0x7f)
    ws = torch.full((256,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    sao.sao_rms_norm_fwd(x, c["weight"], eps, ws, residual=res, scaling=scaling, stream=stream, **o)
    torch.cuda.synchronize()
    return o


def check_forward(c, o, eps=1e-6, scaling="none"):
    x, h = c["x"], c["x"].shape[1]
    r = x
    if c["residual"] is not None:
        exact = x.double() + c["residual"].double()
        assert ((o["sum"].double() - exact).abs() <= (U + half(x)) * exact.abs()).all()
        r = o["sum"]
    r = r.double()
    rstd = (r.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    y = r * rstd * c["weight"].double()
    if o["rstd"] is not None:
        assert ((o["rstd"].double() - rstd[:, 0]).abs() <= 32 * U * rstd[:, 0]).all()
    if o["y"] is not None:
        # below the least normal number a rounding is off by half the least denormal one, however small the value:
        # 2^-150 in fp32 (twice, in a product of three) and, in a bf16 y, 2^-134
        tiny = 2.0 ** -149 + (2.0 ** -134 if o["y"].dtype is torch.bfloat16 else 0.0)
        assert ((o["y"].double() - y).abs() <= (34 * U + half(x)) * y.abs() + tiny).all()
    if scaling == "none":
        return
    size = {"row": h, "block": 128, "mx": 32}[scaling]
    amax = torch.stack([b.abs().amax(1) for b in y.split(size, 1)], 1) / 448
    s = o["scales"].double()
    if scaling == "mx":
        assert (s >= amax * (1 - 40 * U)).all() and ((s / 2 < amax * (1 + 40 * U)) | (s == 2.0 ** -127)).all()
        assert (torch.frexp(s).mantissa == 0.5).all()
    else:
        assert ((s - amax.clamp(min=2.0 ** -126)).abs() <= 40 * U * s).all()
    s = s.repeat_interleave(size, 1)[:, :h]
    got = o["y8"].double() * s
    assert ((got - y).abs() <= (2.0 ** -4 + 40 * U) * y.abs() + 2.0 ** -10 * s).all()


def backward(c, o, dsum=True, dw=True, accumulate=False, offset=0, stream=None, into=None):
    x = o["sum"] if o["sum"] is not None else c["x"]
    N, h = x.shape
    dx = _new(x, offset) if into is None else into
    dweight = (torch.full((h,), 2.0 if accumulate else math.nan, device="cuda") if dw else None)
    ws = sao.norm_workspace(N, h)
    ws.fill_(255)
    torch.cuda.synchronize()
    sao.sao_rms_norm_bwd(x, c["weight"], o["rstd"], c["dy"], dx, dweight, ws, dsum=c["dsum"] if dsum else None,
                         accumulate=accumulate, stream=stream)
    torch.cuda.synchronize()
    return dx, dweight


def check_backward(c, o, dx, dw, dsum=True, accumulate=False, eps=1e-6):
    x = (o["sum"] if o["sum"] is not None else c["x"]).double()
    w, dy = c["weight"].double(), c["dy"].double()
    rstd = (x.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    a = dy * w
    mean = (a * x).mean(1, keepdim=True) * rstd ** 3
    ds = c["dsum"].double() if dsum else torch.zeros_like(x)
    want = ds + rstd * a - x * mean
    size = rstd * a.abs() + x.abs() * (a * x).abs().mean(1, keepdim=True) * rstd ** 3 + ds.abs()
    assert ((dx.double() - want).abs() <= 64 * U * size + half(c["x"]) * want.abs()).all()
    if dw is not None:
        terms = dy * x * rstd
        want = terms.sum(0) + (2.0 if accumulate else 0.0)
        assert ((dw.double() - want).abs() <= 64 * U * terms.abs().sum(0) + 2 * U * want.abs()).all()


SIZES = [(1, 1), (3, 7), (2, 8), (5, 31), (4, 32), (1, 100), (9, 127), (300, 128), (33, 129), (1000, 256), (77, 512), (2001, 515), (152, 1024),
         (153, 1032), (1, 2048), (5000, 2048), (200, 2056), (31, 4099), (700, 4096), (3, 6144), (330, 6144), (170, 8192), (5, 8200),
         (2, 16383), (160, 16383), (7, 16384), (155, 16384)]


@pytest.mark.parametrize("w_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,h", SIZES)
def test_against_fp64(N, h, dtype, w_dtype):
    residual = (N + h) % 3 != 0
    c = _case(N, h, dtype, w_dtype, residual, seed=N + h)
    o = forward(c)
    check_forward(c, o)
    dsum = N % 2 == 1
    check_backward(c, o, *backward(c, o, dsum=dsum), dsum=dsum)


@pytest.mark.parametrize("scaling", ["row", "block", "mx"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,h", SIZES)
def test_eight_bits(N, h, dtype, scaling):
    c = _case(N, h, dtype, residual=N % 2 == 0, seed=N + h + 1)
    check_forward(c, forward(c, scaling=scaling, want_y=h % 2 == 0, rstd=False), scaling=scaling)


@pytest.mark.parametrize("scaling", ["row", "block", "mx"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,h", [(3000, 5), (700, 24), (1001, 47), (400, 64), (333, 129), (90, 771), (61, 2259), (7, 9001)])
def test_eight_bits_beside_y(N, h, dtype, scaling):
    for residual in (True, False):
        c = _case(N, h, dtype, residual=residual, seed=h)
        check_forward(c, forward(c, scaling=scaling), scaling=scaling)


@pytest.mark.parametrize("h", [640, 2048])
@pytest.mark.parametrize("dtype,offset", [("f32", 1), ("f32", 2), ("bf16", 1), ("bf16", 4), ("bf16", 8)])
def test_alignment(dtype, offset, h):
    c = _case(50, h, dtype, offset=offset)
    o = forward(c, scaling="block", offset=offset)
    check_forward(c, o, scaling="block")
    check_backward(c, o, *backward(c, o, offset=offset))


@pytest.mark.parametrize("one", ["x", "residual", "weight", "dy", "dsum"])
def test_one_array_off_16_bytes(one):
    c = _case(40, 512)
    c[one] = _place(c[one].clone(), 1)
    o = forward(c, scaling="mx")
    check_forward(c, o, scaling="mx")
    check_backward(c, o, *backward(c, o))


@pytest.mark.parametrize("h", [96, 99, 515, 1001, 2048])
def test_in_place(h):
    """sum over x, over residual; dx over dy, over dsum; dweight added to; no dweight."""
    for over in ("x", "residual"):
        c = _case(301, h, seed=h)
        d = {k: v.clone() for k, v in c.items()}
        y, rstd, ws = torch.empty_like(c["x"]), torch.empty(301, device="cuda"), sao.norm_workspace(301, h)
        sao.sao_rms_norm_fwd(d["x"], d["weight"], 1e-6, ws, residual=d["residual"], sum=d[over], y=y, rstd=rstd)
        o = {"sum": d[over], "y": y, "rstd": rstd}
        check_forward(c, o)
        for into in ("dy", "dsum"):
            e = {k: v.clone() for k, v in c.items()}
            dx, dw = backward(e, o, accumulate=True, into=e[into])
            check_backward(c, o, dx, dw, accumulate=True)
        dx, dw = backward(c, o, dw=False)
        check_backward(c, o, dx, dw)


@pytest.mark.parametrize("eps", [0.0, 1e-6, 10.0])
def test_small_and_large_rows(eps):
    """Rows of 2^-60 to 2^55, one of zeros (not with eps 0, where it has no norm)."""
    c = _case(40, 1000, "f32", residual=False)
    c["x"] *= torch.exp2(torch.linspace(-60, 54, 40, device="cuda").round())[:, None]
    if eps:
        c["x"][7] = 0
    c["dsum"].zero_()
    o = forward(c, eps)
    check_forward(c, o, eps)
    check_backward(c, o, *backward(c, o, dw=False), eps=eps)


def test_zeros_and_small_blocks_have_a_scale():
    for scaling in ("row", "block", "mx"):
        c = _case(6, 256, residual=False)
        c["x"][0] = 0
        c["x"][1, 100:] = 0
        c["weight"][128:160] = 2.0 ** -140
        o = forward(c, scaling=scaling)
        check_forward(c, o, scaling=scaling)
        assert (o["y8"][0].float() == 0).all() and (o["scales"][0].float() > 0).all()


@pytest.mark.parametrize("h", [99, 512])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_not_finite_stays_in_its_row(what, h):
    c = _case(20, h, residual=False)
    clean = {s: forward(c, scaling=s) for s in ("row", "block", "mx")}
    c["x"][3, 5] = what
    others = [i for i in range(20) if i != 3]
    for s, o in clean.items():
        n = forward(c, scaling=s)
        for k in ("y", "rstd", "y8", "scales"):
            assert torch.equal(n[k][others].float(), o[k][others].float())
        assert math.isnan(n["y"][3, 5].item()) and math.isnan(n["scales"][3, 0].float().item())
    assert forward(c)["rstd"][3].item() == 0 if what == math.inf else True


def test_no_rows():
    x = torch.empty(0, 64, device="cuda")
    w, dw, ws = torch.ones(64, device="cuda"), torch.full((64,), 5.0, device="cuda"), sao.norm_workspace(0, 64)
    r = torch.empty(0, device="cuda")
    sao.sao_rms_norm_fwd(x, w, 1e-6, ws, y=x)
    sao.sao_rms_norm_bwd(x, w, r, x, x, dw, ws, accumulate=True)
    assert (dw == 5).all()
    sao.sao_rms_norm_bwd(x, w, r, x, x, dw, ws)
    assert (dw == 0).all()


def test_against_differences():
    """The gradients of a sum over y and the stream, from the forward's own outputs in fp32."""
    c = _case(3, 40, "f32", seed=4)
    o = forward(c)
    dx, dw = backward(c, o)
    f = lambda: (lambda p: float((p["y"].double() * c["dy"].double()).sum() + (p["sum"].double() * c["dsum"].double()).sum()))(forward(c))
    step = 2.0 ** -8  # the difference's own error: third derivatives by step^2, outputs' roundings (34 u of them) by 1 / step
    for t, g in ((c["x"], dx), (c["weight"], dw)):
        flat = t.view(-1)
        for i in range(0, flat.numel(), 7):
            v = flat[i].item()
            flat[i] = v + step
            up, right = f(), flat[i].item()
            flat[i] = v - step
            down, left = f(), flat[i].item()
            flat[i] = v
            d = (up - down) / (right - left)
            scale = float((o["y"].double() * c["dy"].double()).abs().sum() + (o["sum"].double() * c["dsum"].double()).abs().sum())
            assert abs(d - g.view(-1)[i].item()) <= 34 * U * scale / step + 4 * step ** 2 * scale


def test_repeats_bit_for_bit_and_in_a_graph_and_on_a_stream():
    c = _case(3001, 1024, seed=5)
    outs = []
    for stream in (None, None, torch.cuda.Stream()):
        o = forward(c, scaling="block", stream=stream)
        outs.append([o["sum"], o["y"], o["rstd"], o["y8"].view(torch.uint8), o["scales"], *backward(c, o, stream=stream)])
    assert all(torch.equal(a, b) for later in outs[1:] for a, b in zip(outs[0], later))
    ws, o = sao.norm_workspace(3001, 1024), [torch.empty_like(t) for t in outs[0]]
    s, y, rstd, y8, scales, dx, dw = o
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sao.sao_rms_norm_fwd(c["x"], c["weight"], 1e-6, ws, residual=c["residual"], sum=s, y=y, rstd=rstd, y8=y8,
                             scales=scales, scaling="block")
        sao.sao_rms_norm_bwd(s, c["weight"], rstd, c["dy"], dx, dw, ws, dsum=c["dsum"])
    for _ in range(2):
        for t in o:
            t.view(torch.uint8).fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("N,h", [(100, 264), (99, 515), (101, 1001), (97, 77)])
def test_rows_past_the_last_stay_as_they_were(N, h):
    c = _case(129, h, residual=False)
    big = {k: torch.full((129, h), 7.0, device="cuda", dtype=torch.bfloat16) for k in ("y", "dx")}
    rstd, ws = torch.full((129,), 7.0, device="cuda"), sao.norm_workspace(N, h)
    sao.sao_rms_norm_fwd(c["x"][:N], c["weight"], 1e-6, ws, y=big["y"][:N], rstd=rstd[:N])
    sao.sao_rms_norm_bwd(c["x"][:N], c["weight"], rstd[:N], c["dy"][:N], big["dx"][:N], None, ws)
    assert (rstd[N:] == 7).all() and all((t[N:] == 7).all() for t in big.values())


def test_past_32_bits():
    """More than 2^31 elements: the last rows are as those of a call on them alone."""
    N, h = (1 << 20) + 3, 2048
    x = torch.randn(4, h, generator=torch.Generator().manual_seed(6)).bfloat16().cuda().repeat((N + 3) // 4, 1)[:N].contiguous()
    w, rstd, ws = torch.ones(h, device="cuda"), torch.empty(N, device="cuda"), sao.norm_workspace(N, h)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    sao.sao_rms_norm_fwd(x, w, 1e-6, ws, y=y, rstd=rstd)
    sao.sao_rms_norm_bwd(x, w, rstd, x, dx, None, ws)
    z, r4, d4 = torch.empty_like(x[:4]), torch.empty(4, device="cuda"), torch.empty_like(x[:4])
    sao.sao_rms_norm_fwd(x[:4], w, 1e-6, ws, y=z, rstd=r4)
    sao.sao_rms_norm_bwd(x[:4], w, r4, x[:4], d4, None, ws)
    # two results of one value: twice the bounds of one. With dy = x and a weight of 1, dx is the difference of two terms
    # that are nearly equal, each |x| rstd: 64 u of both and a rounding, of which the value itself may be nothing
    assert N % 4 == 3
    size = 2 * x[:3].double().abs() * r4[:3, None].double()
    for big, small, term in ((y, z, 0.0), (dx, d4, size)):
        apart = (big[-3:].double() - small[:3].double()).abs()
        assert (apart <= 2 * ((34 * U + half(x)) * small[:3].double().abs() + 64 * U * (1 + half(x)) * term) * 1.01).all()
