"""Routing to experts against fp64: choices equal, weights and gradients within bounds.

Bounds with u = 2^-24: an exponential of a difference d is off by (|d| + 3) u of itself, sums of up to 1,024 of them by
another 40 u, quotients and products by a few: (|d| + 50) u of a weight, with |d| at most the span of the row's logits
or, for a sigmoid, their largest magnitude. A gradient has one more sum and two more products: (|d| + 70) u of its terms'
absolute values, and its type's rounding."""
import math

import pytest
import torch

from paper_2607_07508_gb300 import sao
from tests import _route as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -140  # a few roundings below the least normal number
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SCORE = {"softmax": sao.SAO_SCORE_SOFTMAX, "sigmoid": sao.SAO_SCORE_SIGMOID}


def _place(t, offset):
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    return flat[offset:].view(t.shape).copy_(t)


def _logits(N, E, dtype="f32", seed=0, size=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(N, E, generator=g) * size + torch.randn(E, generator=g) * 0.5).to(DT[dtype]).cuda()


def _bias(E, seed=0):
    return (torch.randn(E, generator=torch.Generator().manual_seed(seed + 99)) * 0.1).cuda()


def forward(x, k, score="softmax", bias=None, mask=None, groups=1, kept=1, two=False, renorm=True, scale=2.5, given=None,
            offset=0, stream=None):
    N, E = x.shape
    ids = torch.full((N, k), -7, dtype=torch.int32, device="cuda") if given is None else given.clone()
    ids = _place(ids, offset)
    w = _place(torch.full((N, k), math.nan), offset)
    ws = sao.route_workspace(N, E)
    ws.fill_(255)
    torch.cuda.synchronize()
    sao.sao_route_fwd(x, SCORE[score], ids, w, ws, bias=bias, row_mask=mask, groups=groups, groups_kept=kept,
                      group_score=sao.SAO_GROUP_TOP2 if two else sao.SAO_GROUP_MAX, renormalise=renorm, scale=scale,
                      replay=given is not None, stream=stream)
    torch.cuda.synchronize()
    return ids, w


def backward(x, ids, w, grad, score="softmax", mask=None, renorm=True, scale=2.5, into=None, offset=0, stream=None):
    dx = _place(torch.full(x.shape, math.nan, dtype=x.dtype), offset) if into is None else into
    ws = sao.route_workspace(*x.shape)
    ws.fill_(255)
    torch.cuda.synchronize()
    sao.sao_route_bwd(x, SCORE[score], ids, w, grad, dx, ws, row_mask=mask, renormalise=renorm, scale=scale,
                      accumulate=into is not None, stream=stream)
    torch.cuda.synchronize()
    return dx


def _reach(x, score):
    """|d| of the bounds, by row."""
    f = x.double().masked_fill(~torch.isfinite(x), 0.0)
    return f.abs().amax(1, keepdim=True) if score == "sigmoid" else f.amax(1, keepdim=True) - f.amin(1, keepdim=True)


def check(x, k, score="softmax", bias=None, mask=None, groups=1, kept=1, two=False, renorm=True, scale=2.5, given=None,
          offset=0, seed=0, train=True):
    ids, w = forward(x, k, score, bias, mask, groups, kept, two, renorm, scale, given, offset)
    N, E = x.shape
    on = R.usable(x, score)
    if mask is not None:
        on = on & (mask != 0)
    if given is None:
        want = torch.where(on[:, None], R.choose(x, k, score, bias, groups, kept, two), -1)
        wrong = (ids != want).any(1)
        assert not wrong.any(), (int(wrong.sum()), ids[wrong][:2].tolist(), want[wrong][:2].tolist())
    else:
        assert torch.equal(ids, given)
    want_w = R.weights(x, ids, score, renorm, scale, on)
    tol = (_reach(x, score) + 50) * U
    assert ((w.double() - want_w).abs() <= tol * want_w.abs() + TINY).all()
    if not train:
        return ids, w
    grad = torch.randn(N, k, generator=torch.Generator().manual_seed(seed)).cuda()
    want, size = R.gradient(x, ids, want_w, grad, score, renorm, scale, on)
    half = torch.finfo(x.dtype).eps / 2
    tol = (_reach(x, score) + 70) * U
    dx = backward(x, ids, w, grad, score, mask, renorm, scale, offset=offset)
    assert ((dx.double() - want).abs() <= tol * size + half * want.abs() + TINY).all()
    before = _logits(N, E, seed=seed + 1).to(x.dtype)
    dx = backward(x, ids, w, grad, score, mask, renorm, scale, into=before.clone())
    want = want + before.double()
    assert ((dx.double() - want).abs() <= tol * size + (half + U) * want.abs() + TINY).all()
    return ids, w


SIZES = [(1, 1, 1), (1, 8, 2), (3, 4, 4), (2, 7, 7), (31, 33, 3), (33, 32, 8), (257, 100, 4), (513, 128, 8), (1000, 63, 6),
         (300, 160, 8), (129, 256, 8), (40, 257, 10), (77, 512, 1), (65, 1000, 32), (20, 1024, 32), (4001, 64, 6), (5, 48, 32)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,E,k", SIZES)
def test_against_fp64(N, E, k, dtype, score):
    x = _logits(N, E, dtype, seed=N + E)
    for bias in (None, _bias(E)):
        for renorm in (True, False):
            check(x, k, score, bias, renorm=renorm, seed=k)


GROUPS = [(40, 2, 1, 5), (64, 4, 3, 8), (256, 8, 4, 8), (160, 8, 3, 6), (160, 5, 2, 10), (96, 16, 2, 7), (32, 32, 9, 9),
          (544, 17, 4, 12), (1023, 31, 30, 32), (1024, 32, 2, 16), (12, 3, 3, 12), (6, 6, 2, 2), (510, 10, 7, 3)]


@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,groups,kept,k", GROUPS)
def test_groups(E, groups, kept, k, dtype, score, two):
    x = _logits(333, E, dtype, seed=E + groups)
    for bias in (None, _bias(E)):
        check(x, k, score, bias, groups=groups, kept=kept, two=two, renorm=bias is None)


# With many tokens rows are taken by eight lanes each, up to 512 experts and eight a token.
MANY = [(16, 1, 1, 1), (17, 1, 1, 5), (63, 1, 1, 6), (64, 1, 1, 8), (96, 2, 1, 3), (100, 4, 3, 8), (128, 1, 1, 8),
        (160, 8, 3, 8), (256, 8, 4, 8), (256, 2, 1, 7), (257, 1, 1, 8), (384, 4, 1, 2), (512, 8, 7, 8), (24, 8, 2, 6)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,groups,kept,k", MANY)
def test_many_tokens(E, groups, kept, k, dtype, score):
    N = 5003
    x = _logits(N, E, dtype, seed=E + k)
    mask = (torch.rand(N, generator=torch.Generator().manual_seed(E)) < 0.7).to(torch.uint8).cuda()
    for bias in (None, _bias(E), _bias(E) * 30 - 100):
        for two in (False, True) if groups > 1 else (False,):
            check(x, k, score, bias, mask if E % 2 else None, groups, kept, two, renorm=two or bias is None or k == 6)
    check(x, k, score, None, mask, groups, kept, False, renorm=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,E,k", [(45001, 40, 8), (50000, 63, 5), (160003, 96, 8), (165000, 129, 2), (165000, 256, 8)])
def test_a_great_many_tokens(N, E, k, dtype, score):
    """A thread to a row of more than 32 experts; copies that differ in their last bits among them."""
    g = torch.Generator().manual_seed(E)
    x = torch.randn(N, (E + 1) // 2, generator=g).repeat(1, 2)[:, :E].contiguous()
    x = (x.view(torch.int32) + torch.randint(-3, 4, (N, E), generator=g, dtype=torch.int32)).view(torch.float32)
    x = torch.where((torch.arange(N) % 3 == 0)[:, None], x, torch.randn(N, E, generator=g)).to(DT[dtype]).cuda()
    x[::1000, 3], x[1::1000, 5], x[2::1000], x[3::1000, 1:] = math.nan, math.inf, -math.inf, -math.inf
    bias = _bias((E + 1) // 2).repeat(2)[:E].contiguous()
    for b in (None, bias):
        check(x, k, score, b, train=False)
    check(x, k, score, None, renorm=False, train=False)
    check(x, k, score, torch.zeros(E, device="cuda"), (torch.arange(N) % 5 != 0).to(torch.uint8).cuda(), train=False)


# Up to 32 experts in one group, eight a token: a thread to a row.
FEW = [(1, 1), (2, 1), (5, 2), (8, 2), (8, 8), (9, 3), (15, 5), (16, 4), (17, 8), (23, 7), (31, 1), (32, 8)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,k", FEW)
def test_few_experts(E, k, dtype, score):
    N = 9001
    x = _logits(N, E, dtype, seed=E + k)
    mask = (torch.rand(N, generator=torch.Generator().manual_seed(E)) < 0.7).to(torch.uint8).cuda()
    for bias in (None, _bias(E), _bias(E) * 30 - 100):
        for renorm in (True, False):
            check(x, k, score, bias, mask if renorm else None, renorm=renorm)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,groups,kept,k", [(2, 2, 1, 1), (6, 3, 2, 1), (8, 2, 1, 4), (16, 16, 11, 8), (20, 4, 1, 2), (24, 8, 3, 6),
                                             (27, 9, 4, 5), (28, 4, 2, 3), (30, 5, 2, 8), (32, 4, 3, 8), (32, 32, 9, 8)])
def test_few_experts_in_groups(E, groups, kept, k, dtype, score):
    N = 6007
    g = torch.Generator().manual_seed(E)
    x = torch.randn(N, (E + 1) // 2, generator=g).repeat(1, 2)[:, :E].contiguous()
    x = (x.view(torch.int32) + torch.randint(-3, 4, (N, E), generator=g, dtype=torch.int32)).view(torch.float32)
    x = torch.where((torch.arange(N) % 2 == 0)[:, None], x, torch.randn(N, E, generator=g) * 2).to(DT[dtype]).cuda()
    x[::50, 1], x[1::50, 0], x[2::50, :E // 2], x[3::50, 1:] = math.nan, math.inf, -math.inf, -math.inf
    bias = _bias((E + 1) // 2).repeat(2)[:E].contiguous()
    out = _bias(E, seed=1)
    out[::3] = -math.inf
    for b in (None, bias, torch.zeros(E, device="cuda"), out):
        for two in (False, True):
            check(x, k, score, b, None, groups, kept, two, renorm=not two, train=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,k", [(6, 2), (16, 8), (30, 5)])
def test_few_experts_of_near_and_extraordinary_keys(E, k, dtype, score):
    """Copies that differ in their last bits, few different logits, NaN, infinities, the lowest value, biases that are out."""
    N, inf = 6000, math.inf
    g = torch.Generator().manual_seed(E)
    x = torch.randn(N, (E + 1) // 2, generator=g).repeat(1, 2)[:, :E].contiguous()
    x = (x.view(torch.int32) + torch.randint(-3, 4, (N, E), generator=g, dtype=torch.int32)).view(torch.float32)
    few = torch.randint(0, 3, (N, E), generator=g).float() * 0.3
    x = torch.where((torch.arange(N) % 3 == 0)[:, None], few, x).to(DT[dtype]).cuda()
    kind = torch.randint(0, 12, (N,), generator=g).cuda()
    x[kind == 0, 1], x[kind == 1, 2], x[kind == 2, 0] = math.nan, inf, -inf
    x[kind == 3], x[kind == 4, 1:] = -inf, -inf
    x[kind == 5, 2:] = torch.finfo(x.dtype).min
    x[kind == 6] *= 60
    bias = _bias((E + 1) // 2).repeat(2)[:E].contiguous()
    out = bias.clone()
    out[1], out[3] = -inf, math.nan
    top = bias.clone()
    top[2] = inf
    for b in (None, bias, torch.zeros(E, device="cuda"), out, bias * 1e6, top):
        check(x, k, score, b, renorm=True, train=False)
        check(x[:5000].contiguous(), k, score, b, renorm=False, train=False)


@pytest.mark.parametrize("k", [8, 5])
@pytest.mark.parametrize("groups,kept,two", [(1, 1, False), (8, 3, False), (8, 3, True), (2, 1, True)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N", [700, 4000])
def test_equal_and_near_keys(N, score, groups, kept, two, k):
    """Few different logits; logits that differ in their last bits; keys with a bias that differ by its rounding."""
    E = 128
    g = torch.Generator().manual_seed(k)
    for levels in (1, 3, 40):
        x = (torch.randint(0, levels, (N, E), generator=g).float() * 0.3 - 0.6).cuda()
        for dtype in ("f32", "bf16"):
            for bias in (None, torch.zeros(E, device="cuda"), (torch.randint(0, 2, (E,), generator=g) * 0.25).cuda()):
                check(x.to(DT[dtype]), k, score, bias, groups=groups, kept=kept, two=two, train=False)
    base = _logits(1, E, seed=3).repeat(N, 1)
    moved = (base.view(torch.int32) + torch.randint(-40, 40, (N, E), generator=g, dtype=torch.int32).cuda()).view(torch.float32)
    x = torch.where(torch.rand(N, E, generator=g).cuda() < 0.5, moved, base[:, :1]).contiguous()
    bias = (0.75 - R.scores(base[:1].double(), score)[0]).float()
    near = torch.where(torch.rand(N, E, generator=g).cuda() < 0.5, moved, base).contiguous()
    for rows, b in ((x, None), (moved, None), (near, bias)):
        check(rows, k, score, b, groups=groups, kept=kept, two=two, train=False)


@pytest.mark.parametrize("k", [1, 3, 4, 7, 8])
@pytest.mark.parametrize("groups,kept,two", [(1, 1, False), (4, 3, False), (8, 5, True)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N", [900, 4000])
def test_experts_in_pairs(N, score, groups, kept, two, k):
    """Experts in pairs, or threes, whose logits differ by a few of their last bits, one or the other of them the larger:
    the last choice falls between such, or within a group that is such a copy of another."""
    E = 96
    g = torch.Generator().manual_seed(k)
    for copies in (2, 3):
        x = (torch.randn(N, E // copies, generator=g) * 1.5).cuda().repeat(1, copies)
        x = (x.view(torch.int32) + torch.randint(-6, 7, (N, E), generator=g, dtype=torch.int32).cuda()).view(torch.float32)
        bias = _bias(E // copies, seed=copies).repeat(copies)
        order = torch.randperm(E, generator=g).cuda()
        for b in (None, bias):
            check(x.contiguous(), k, score, b, groups=groups, kept=kept, two=two, train=False)
            check(x[:, order].contiguous(), k, score, None if b is None else b[order].contiguous(), groups=groups, kept=kept,
                  two=two, train=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups,kept", [(1, 1), (4, 2)])
@pytest.mark.parametrize("N", [300, 3000])
def test_rows_out_of_the_ordinary(N, groups, kept, dtype, score):
    """NaN, infinities, rows with few experts or none, the type's lowest value, far and large logits, biases that are out."""
    E, inf = 64, math.inf
    x = _logits(N, E, dtype, seed=21)
    g = torch.Generator().manual_seed(22)
    kind = torch.randint(0, 12, (N,), generator=g).cuda()
    at = torch.randint(0, E, (N,), generator=g).cuda()
    x[torch.arange(N).cuda(), at] = torch.where(kind < 3, torch.tensor([math.nan, inf, -inf]).cuda()[kind.clamp(max=2)],
                                                x[torch.arange(N).cuda(), at].float()).to(x.dtype)
    x[kind == 3] = -inf
    x[kind == 4, 3:] = -inf
    x[kind == 5, 2:] = torch.finfo(x.dtype).min
    x[kind == 6] *= 40
    x[kind == 7] -= 200
    x[kind == 8] *= 1e30
    bias = _bias(E)
    bias[5], bias[6] = -inf, math.nan
    large = bias.clone()
    large[9] = 1e4
    top = bias.clone()
    top[9] = inf
    for b in (None, bias, large, top):
        for two in (False, True):
            check(x, 6, score, b, groups=groups, kept=kept, two=two, renorm=True, train=False)
    check(x, 8, score, None, groups=groups, kept=kept, renorm=False, train=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("levels", [1, 2, 3, 40])
@pytest.mark.parametrize("groups,kept", [(1, 1), (8, 3), (16, 5)])
def test_equal_logits_go_by_the_lower_index(groups, kept, levels, score):
    """Few different logits, -0 and 0 among them, without a bias, with one of zeros and one of few different values."""
    g = torch.Generator().manual_seed(levels)
    x = (torch.randint(0, levels, (200, 96), generator=g).float() * 0.5).cuda()
    x[::2] = torch.where(x[::2] == 0, -0.0, x[::2])
    few = (torch.randint(0, 2, (96,), generator=g).float() * 0.25).cuda()
    for bias in (None, torch.zeros(96, device="cuda"), few):
        for two in (False, True):
            check(x, 6, score, bias, groups=groups, kept=kept, two=two)


@pytest.mark.parametrize("groups,kept,two", [(1, 1, False), (8, 2, False), (8, 2, True)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_keys_that_fp32_cannot_tell_apart(score, groups, kept, two):
    """Biases that make all keys of a row equal but for the biases' rounding, 3e-8; some logits of other rows moved by
    as little as fp32 has."""
    E = 128
    x = _logits(1, E, seed=3).repeat(300, 1)
    bias = (0.75 - R.scores(x[:1].double(), score)[0]).float()
    g = torch.Generator().manual_seed(5)
    move = torch.randint(-2, 3, (300, E), generator=g, dtype=torch.int32).cuda()
    moved = (x.view(torch.int32) + move).view(torch.float32)
    x = torch.where(torch.rand(300, E, generator=g).cuda() < 0.3, moved, x).contiguous()
    check(x, 8, score, bias, groups=groups, kept=kept, two=two)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_far_logits(score):
    """Scores that vanish or are 1 to any precision: without a bias the logits decide."""
    x = _logits(300, 64, seed=8, size=60.0)
    check(x, 8, score)
    check(x, 8, score, _bias(64))
    check(x, 8, score, renorm=False)
    check(x - 300, 8, score)
    check(x + 300, 8, score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(1, 1), (4, 2)])
def test_experts_that_are_out(groups, kept, score):
    """Logits of -inf, rows with fewer than k experts or none, biases of -inf, NaN and inf."""
    E, inf, nan = 32, math.inf, math.nan
    x = _logits(64, E, seed=9)
    x[:, 3] = -inf
    x[1, 4:] = -inf
    x[2] = -inf
    x[3, 1:] = -inf
    x[4, ::2] = -inf
    x[5, 8:16] = -inf
    x[5, 9] = 1.0
    bias = _bias(E)
    bias[5], bias[6], bias[20] = -inf, nan, inf
    for b in (None, bias):
        for two in (False, True):
            for renorm in (True, False):
                check(x, 7, score, b, groups=groups, kept=kept, two=two, renorm=renorm)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("replay", [True, False])
def test_rows_without_scores(replay, renorm, score):
    x = _logits(40, 48, seed=10)
    x[3, 7] = math.nan
    x[4] = math.nan
    x[5, 40] = math.inf
    x[6] = -math.inf
    x[7, 2] = -math.nan
    given = R.choose(_logits(40, 48, seed=10), 4, score) if replay else None
    ids, w = check(x, 4, score, renorm=renorm, given=given)
    assert (w[[3, 4, 6, 7]] == 0).all() and (replay or (ids[[3, 4, 6, 7]] == -1).all())
    sao.sao_set_checked(True)
    try:
        for rows, bad in ((x, True), (x[6:7], False)):
            i, ws = torch.empty(len(rows), 4, dtype=torch.int32, device="cuda"), sao.route_workspace(len(rows), 48)
            v = torch.empty(len(rows), 4, device="cuda")
            call = lambda: sao.sao_route_fwd(rows, SCORE[score], i, v, ws)
            if bad:
                with pytest.raises(sao.SaoError, match="logits-without-scores"):
                    call()
            else:
                call()
    finally:
        sao.sao_set_checked(False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 5, 1000])
def test_masked_rows(N, dtype, score):
    x = _logits(N, 96, dtype, seed=11)
    mask = (torch.arange(N) % 3 == 1).to(torch.uint8).cuda()
    x[mask == 0] = math.nan
    for renorm in (True, False):
        check(x, 8, score, _bias(96), mask, groups=8, kept=4, two=True, renorm=renorm)
    check(x, 8, score, mask=torch.zeros_like(mask))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("N,E,k", [(500, 60, 9), (6001, 60, 8), (6001, 24, 5), (40000, 60, 4), (9001, 6, 8)])
def test_replay(N, E, k, renorm, dtype, score):
    """A rollout's choices: others than the logits', the same expert twice, some of them missing, rows of none."""
    x = _logits(N, E, dtype, seed=12)
    g = torch.Generator().manual_seed(12)
    k = min(k, E)
    given = torch.randint(-1, E, (N, k), generator=g, dtype=torch.int32).cuda()
    given[7], given[8], given[9, 1:] = -1, E - 1, -(1 << 31)
    x[10, 5], x[11, 3], x[12] = -math.inf, math.nan, -math.inf
    given[10] = 5
    mask = (torch.rand(N, generator=g) < 0.8).to(torch.uint8).cuda()
    check(x, k, score, mask=mask, renorm=renorm, given=given)
    check(x, k, score, mask=None, renorm=renorm, given=given)


@pytest.mark.parametrize("N", [20, 6000])
def test_ids_past_the_last_expert(N):
    x = _logits(N, 16)
    given = torch.full((N, 3), 15, dtype=torch.int32, device="cuda")
    given[4, 1], given[5, 2] = 16, (1 << 31) - 1
    ids, w = check(x, 3, given=given)
    assert w[4, 1] == 0 and w[5, 2] == 0 and (w[4, [0, 2]] == 1.25).all()
    sao.sao_set_checked(True)
    try:
        for call in (lambda: forward(x, 3, given=given), lambda: backward(x, given, w, w)):
            with pytest.raises(sao.SaoError, match="expert-id"):
                call()
    finally:
        sao.sao_set_checked(False)


@pytest.mark.parametrize("scale", [0.0, 1.0, -2.0, 1e-30])
def test_scales(scale):
    x = _logits(50, 40, seed=13)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            check(x, 4, score, scale=scale, renorm=renorm)


@pytest.mark.parametrize("E", [40, 63, 64, 128, 256])
@pytest.mark.parametrize("dtype,offset", [("f32", 1), ("f32", 2), ("bf16", 1), ("bf16", 2), ("bf16", 4)])
def test_alignment(dtype, offset, E):
    x = _place(_logits(301, E, dtype, seed=14), offset)
    check(x, 5, "sigmoid", _bias(E), offset=offset)
    check(x, 5, "softmax", renorm=False, offset=offset)


def test_against_differences():
    """Gradients of a sum over weights, from the forward in fp32 with its choices given."""
    x = _logits(4, 12, seed=15)
    grad = torch.randn(4, 5, generator=torch.Generator().manual_seed(1)).cuda()
    step = 2.0 ** -7
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            ids, w = forward(x, 5, score, renorm=renorm)
            dx = backward(x, ids, w, grad, score, renorm=renorm)
            size = float((w.double() * grad.double()).abs().sum())
            f = lambda: float((forward(x, 5, score, renorm=renorm, given=ids)[1].double() * grad.double()).sum())
            for i in range(x.numel()):
                flat, v = x.view(-1), x.view(-1)[i].item()
                flat[i] = v + step
                up, right = f(), flat[i].item()
                flat[i] = v - step
                down, left = f(), flat[i].item()
                flat[i] = v
                # third derivatives of products of scores are below 8 of them; two weights' errors over 2 steps
                assert abs((up - down) / (right - left) - dx.view(-1)[i].item()) <= (60 * U / step + 2 * step ** 2) * size


def test_no_rows():
    x = torch.empty(0, 16, device="cuda")
    ids, w = torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda")
    ws = sao.route_workspace(0, 16)
    sao.sao_route_fwd(x, 0, ids, w, ws)
    sao.sao_route_bwd(x, 0, ids, w, w, x, ws)


def test_repeats_bit_for_bit_and_in_a_graph_and_on_a_stream():
    x, bias = _logits(5003, 160, "bf16", seed=16), _bias(160)
    grad = torch.randn(5003, 8, generator=torch.Generator().manual_seed(2)).cuda()
    outs = []
    for stream in (None, None, torch.cuda.Stream()):
        ids, w = forward(x, 8, "sigmoid", bias, groups=8, kept=3, two=True, stream=stream)
        outs.append((ids, w, backward(x, ids, w, grad, "sigmoid", stream=stream)))
    assert all(torch.equal(a, b) for later in outs[1:] for a, b in zip(outs[0], later))
    o, ws = [torch.empty_like(t) for t in outs[0]], sao.route_workspace(5003, 160)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sao.sao_route_fwd(x, SCORE["sigmoid"], o[0], o[1], ws, bias=bias, groups=8, groups_kept=3,
                          group_score=sao.SAO_GROUP_TOP2, scale=2.5)
        sao.sao_route_bwd(x, SCORE["sigmoid"], o[0], o[1], grad, o[2], ws, scale=2.5)
    for _ in range(2):
        for t in o:
            t.view(torch.uint8).fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("E", [60, 64, 63])
def test_rows_past_the_last_stay_as_they_were(E):
    x = _logits(80, E, "bf16", seed=17)
    N = 37
    ids, w = torch.full((80, 4), 9, dtype=torch.int32, device="cuda"), torch.full((80, 4), 9.0, device="cuda")
    dx = torch.full_like(x, 9)
    ws = sao.route_workspace(N, E)
    sao.sao_route_fwd(x[:N], 0, ids[:N], w[:N], ws)
    for renorm in (True, False):
        sao.sao_route_bwd(x[:N], 0, ids[:N], w[:N], w[:N], dx[:N], ws, renormalise=renorm)
    torch.cuda.synchronize()
    assert (ids[N:] == 9).all() and (w[N:] == 9).all() and (dx[N:] == 9).all()


def test_past_32_bits():
    """More than 2^31 logits: the last rows are those of a call on them alone."""
    N, E = (1 << 21) + 5, 1024
    x = _logits(1 << 11, E, "bf16").repeat(N // (1 << 11) + 1, 1)[:N].contiguous()
    ids, w = torch.empty(N, 2, dtype=torch.int32, device="cuda"), torch.empty(N, 2, device="cuda")
    ws = sao.route_workspace(N, E)
    sao.sao_route_fwd(x, 0, ids, w, ws, scale=2.5)
    a, b = forward(x[-300:].contiguous(), 2)
    assert torch.equal(ids[-300:], a) and torch.equal(w[-300:], b)
    for renorm in (True, False):
        dx = torch.empty_like(x)
        sao.sao_route_bwd(x, 0, ids, w, w, dx, ws, renormalise=renorm, scale=2.5)
        assert torch.equal(dx[-300:], backward(x[-300:].contiguous(), a, b, b, renorm=renorm))
        del dx
