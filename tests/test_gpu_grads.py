"""Global gradient norm and clipping against fp64.

Bounds with u = 2^-24: 64 squares are summed in fp32 (each square, and 9 additions one after another: 10 u of a batch at
most), batches in fp64, and a square root halves that: 5 u, and one rounding to fp32; coef 5 u and one rounding; an element
coef's 6 u and a rounding to its type."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def _grads(shapes, seed=0, size=1.0, offset=0):
    """Tensors of (elements, type), `offset` elements behind 16 bytes."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for n, dt in shapes:
        t = torch.empty(n + offset, dtype=dt, device="cuda")[offset:]
        out.append(t.copy_(torch.randn(n, generator=g) * size))
    return out


def _norm(grads):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in grads))


def _out():
    return (torch.full((1,), -3.0, dtype=torch.float64, device="cuda"), torch.full((1,), -3.0, device="cuda"),
            torch.full((1,), -3.0, device="cuda"))


def run(grads, limit, out=None, stream=None):
    ws = sao.grad_workspace()
    ws.fill_(255)
    sumsq, norm, coef = _out()
    torch.cuda.synchronize()
    sao.sao_grad_sumsq(grads, sumsq, ws, stream=stream)
    sao.sao_grad_clip(grads, sumsq, limit, norm, coef, ws, out=out, stream=stream)
    torch.cuda.synchronize()
    return sumsq.item(), norm.item(), coef.item()


def close(grads, limit, result, out):
    want = _norm(grads)
    sumsq, norm, coef = result
    assert abs(math.sqrt(sumsq) - want) <= 5 * U * want
    assert abs(norm - want) <= 6 * U * want
    c = limit / want if want > limit else 1.0
    assert abs(coef - c) <= 6 * U * c
    for g, o in zip(grads, out):
        d = g.double() * c
        half = torch.finfo(o.dtype).eps / 2  # of a step, relative to the value
        assert ((o.double() - d).abs() <= (7 * U + half) * d.abs() + 2.0 ** -134).all()


MIXED = [(70001, F32), (1, BF16), (0, F32), (8192, F32), (8193, F32), (16384, BF16), (16385, BF16), (7, F32), (0, BF16),
         (31, BF16), (400003, BF16)]


@pytest.mark.parametrize("limit", [0.1, 50.0, 1e6, math.inf])
@pytest.mark.parametrize("offset", [0, 1, 2])
@pytest.mark.parametrize("shapes", [[(1, F32)], [(1, BF16)], [(513, F32)], [(5, F32), (3, BF16)], MIXED])
def test_against_fp64(shapes, offset, limit):
    grads = _grads(shapes, seed=len(shapes), offset=offset)
    out = [torch.full((n + offset,), math.nan, dtype=dt, device="cuda")[offset:] for n, dt in shapes]
    before = [t.clone() for t in grads]
    close(grads, limit, run(grads, limit, out), out)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


@pytest.mark.parametrize("limit", [0.5, 1e6])
def test_in_place(limit):
    grads = _grads(MIXED, seed=3)
    before = [t.clone() for t in grads]
    result = run(grads, limit)
    close(before, limit, result, grads)
    if limit == 1e6:
        assert result[2] == 1.0 and all(torch.equal(a, b) for a, b in zip(grads, before))


def test_out_may_be_the_gradient_or_of_the_other_type():
    grads = _grads([(1000, F32), (70000, BF16), (33, F32), (4096, F32)], seed=4)
    before = [t.clone() for t in grads]
    out = [grads[0], torch.empty(70000, device="cuda"), torch.empty(33, dtype=BF16, device="cuda"),
           torch.empty(4096, dtype=BF16, device="cuda")]
    close(before, 2.0, run(grads, 2.0, out), out)
    assert all(torch.equal(a, b) for a, b in zip(grads[1:], before[1:]))


@pytest.mark.parametrize("count", [47, 48, 49, 511, 512, 513, 1300])
def test_many_tensors(count):
    """Lists that one launch holds and longer ones, small tensors and large ones among them."""
    shapes = [((i * 37) % 900 + (50000 if i % 100 == 99 else 0), BF16 if i % 3 else F32) for i in range(count)]
    grads = _grads(shapes, seed=count)
    out = [torch.full_like(t, math.nan) for t in grads]
    close(grads, 1.5, run(sao.TensorList(grads), 1.5, sao.TensorList(out)), out)


def test_no_tensors():
    for grads in ([], [torch.empty(0, device="cuda")]):
        assert run(grads, 1.0) == (0.0, 0.0, 1.0)
        assert run(grads, 1.0, [torch.empty_like(t) for t in grads]) == (0.0, 0.0, 1.0)


@pytest.mark.parametrize("size", [1e-30, 3e-39, 1e18, 1e35])
def test_squares_past_the_range_of_fp32(size):
    grads = _grads([(5000, F32), (4096, F32), (9, F32)], seed=5, size=size)
    out = [torch.empty_like(t) for t in grads]
    limit = size * 3
    close(grads, limit, run(grads, limit, out), out)


def test_one_large_element_among_small_ones():
    g = _grads([(100000, F32)], size=1e-3)
    g[0][77777] = 3e30
    assert abs(run(g, math.inf)[1] / 3e30 - 1) <= 6 * U


@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_not_finite(what):
    grads = _grads([(5000, F32), (300, BF16)], seed=6)
    grads[1][17] = what
    out = [torch.zeros_like(t) for t in grads]
    sumsq, norm, coef = run(grads, 1.0, out)
    assert not math.isfinite(sumsq) and not math.isfinite(norm) and math.isnan(coef)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(grads, out))


def test_norm_past_the_range_of_fp32():
    g = [torch.full((1 << 20,), 3e38, device="cuda")]
    sumsq, norm, coef = run(g, 1.0)
    want = float(torch.tensor(3e38).double()) * 1024
    assert norm == math.inf and abs(coef * want - 1) <= 2 ** -8  # (a coef below the least normal number)


def test_sums_of_ranks_add_up():
    """Two ranks' shards of the gradients: their sums of squares added give the norm of all."""
    grads = _grads(MIXED, seed=8)
    ws, (a, norm, coef) = sao.grad_workspace(), _out()
    b = torch.empty_like(a)
    sao.sao_grad_sumsq(grads[:4], a, ws)
    sao.sao_grad_sumsq(grads[4:], b, ws)
    a += b
    sao.sao_grad_clip(grads[:4], a, 0.25, norm, coef, ws)
    torch.cuda.synchronize()
    assert abs(norm.item() - _norm(_grads(MIXED, seed=8))) <= 6 * U * norm.item()


def test_repeats_bit_for_bit_and_in_a_graph_and_on_a_stream():
    grads = _grads(MIXED + [(3000000, F32)], seed=9)
    lists = sao.TensorList(grads), sao.TensorList([torch.empty_like(t) for t in grads])
    first = run(lists[0], 1.0, lists[1])
    want = [t.clone() for t in lists[1].tensors]
    assert run(lists[0], 1.0, lists[1], stream=torch.cuda.Stream()) == first
    ws, (sumsq, norm, coef) = sao.grad_workspace(), _out()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sao.sao_grad_sumsq(lists[0], sumsq, ws)
        sao.sao_grad_clip(lists[0], sumsq, 1.0, norm, coef, ws, out=lists[1])
    for _ in range(3):
        for t in lists[1].tensors:
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert (sumsq.item(), norm.item(), coef.item()) == first
        assert all(torch.equal(a, b) for a, b in zip(lists[1].tensors, want))


def test_past_32_bits():
    """More than 2^31 elements and 2^32 bytes in one tensor."""
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[-1], g[1 << 30] = 3.0, 4.0
    _, norm, coef = run([g], 1.0)
    assert abs(norm - 5) <= 6 * U * 5 and abs(coef - 0.2) <= 6 * U
    assert g[-1].item() == torch.tensor(0.6, dtype=BF16).item() and g[1 << 30].item() == torch.tensor(0.8, dtype=BF16).item()
    assert int((g != 0).sum()) == 2
