"""Load-balance loss against fp64.

Bounds with u = 2^-24: a probability is off by at most 16 u of itself (an
exponential, the sum's terms, a quotient); a sum of n of them by another n u at
worst and by sqrt(n) u on random values, so (16 + 4 sqrt(n)) u; the loss the same.
A gradient s (w - sum s w) cancels: 32 u s max |w| absolute, and 2^-8 of itself
where it is written in bf16."""
import numpy as np
import pytest
import torch

from oracle import sao_oracle as O
from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SCORE = {"softmax": 0, "sigmoid": 1}


def _case(N, E, k, dtype="f32", seed=0, lens=None, mask=True):
    g = torch.Generator().manual_seed(seed)
    r = np.random.Generator(np.random.PCG64(seed))
    x = (torch.randn(N, E, generator=g) * 2).to(DT[dtype])
    ids = np.argsort(-x.double().numpy() + r.normal(size=(N, E)), axis=1)[:, :k].astype(np.int32)
    m = (r.random(N) < 0.75).astype(np.uint8) if mask else None
    cu = None if lens is None else np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return x, np.ascontiguousarray(ids), m, cu


def run(x, ids, score, m=None, cu=None, grad=1.0, offset=0, stream=None, fwd_only=False):
    N, E = x.shape
    B = 1 if cu is None else len(cu) - 1
    flat = torch.empty(N * E + offset, dtype=x.dtype, device="cuda")
    xd = flat[offset:].view(N, E)
    xd.copy_(x)
    out = torch.empty(N * E + offset, dtype=x.dtype, device="cuda").fill_(float("nan"))
    dx = out[offset:].view(N, E)
    idd = torch.from_numpy(ids).cuda()
    md = None if m is None else torch.from_numpy(m).cuda()
    cud = None if cu is None else torch.from_numpy(cu).cuda()
    loss = torch.full((1,), float("nan"), device="cuda")
    sums = torch.full((B, E), float("nan"), device="cuda")
    counts = torch.full((B, E), -5, dtype=torch.int64, device="cuda")
    rows = torch.full((B,), -5, dtype=torch.int64, device="cuda")
    ws = sao.balance_workspace(N, E, B)
    ws.fill_(255)
    g = torch.full((1,), grad, device="cuda")
    torch.cuda.synchronize()  # `stream` does not wait for the one that the inputs were made on
    sao.sao_balance_loss_fwd(xd, idd, SCORE[score], loss, counts, sums, rows, ws, row_mask=md, cu_seqlens=cud,
                             stream=stream)
    if not fwd_only:
        sao.sao_balance_loss_bwd(xd, ids.shape[1], SCORE[score], counts, rows, g, dx, ws, row_mask=md, cu_seqlens=cud,
                                 stream=stream)
    torch.cuda.synchronize()
    return {"loss": loss.item(), "counts": counts.cpu().numpy(), "sums": sums.double().cpu().numpy(),
            "rows": rows.cpu().numpy(), "dlogits": dx.double().cpu().numpy()}


def close(got, ref, grad, bf16):
    assert np.array_equal(got["counts"], ref["counts"]) and np.array_equal(got["rows"], ref["rows"])
    rel = (16 + 4 * np.sqrt(ref["rows"].max(initial=1))) * U
    assert (np.abs(got["sums"] - ref["sums"]) <= rel * ref["sums"] + 1e-37).all()
    assert abs(got["loss"] - ref["loss"]) <= rel * ref["loss"]
    d = ref["dlogits"] * grad
    tol = 32 * U * ref["s"] * np.abs(ref["w"]).max(1, initial=0, keepdims=True) * abs(grad)
    assert (np.abs(got["dlogits"] - d) <= tol + (2.0 ** -8 * np.abs(d) if bf16 else 0) + 1e-37).all()


SIZES = [(4096, 32, 2), (4097, 32, 2), (1024, 128, 4), (1025, 128, 4), (1, 1, 1), (1, 8, 2), (2, 7, 7), (31, 33, 3), (32, 64, 8), (257, 100, 4), (1000, 128, 8), (700, 160, 6),
         (65, 256, 8), (40, 1000, 10), (33, 1024, 1), (5000, 8, 2), (20011, 16, 4)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,E,k", SIZES)
def test_batch_against_fp64(N, E, k, dtype, score):
    x, ids, m, _ = _case(N, E, k, dtype, seed=N + E, mask=N > 2)
    ref = O.balance_loss(x, ids, score, m)
    close(run(x, ids, score, m, grad=0.5), ref, 0.5, dtype == "bf16")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [6, 63, 96, 256])
def test_trajectories_against_fp64(E, dtype, score):
    """Empty, one-token, masked and long trajectories, ends inside and at the ends of chunks."""
    lens = [0, 1, 1, 0, 0, 37, 64, 128, 3, 700, 0, 32, 32, 31, 1, 0]
    x, ids, m, cu = _case(sum(lens), E, 3, dtype, seed=E, lens=lens)
    m[cu[6]:cu[7]] = 0
    ref = O.balance_loss(x, ids, score, m, cu)
    close(run(x, ids, score, m, cu), ref, 1.0, dtype == "bf16")


def test_many_short_trajectories():
    r = np.random.Generator(np.random.PCG64(3))
    lens = r.integers(0, 5, 9000)
    x, ids, m, cu = _case(int(lens.sum()), 20, 2, seed=4, lens=lens)
    close(run(x, ids, "softmax", m, cu), O.balance_loss(x, ids, "softmax", m, cu), 1.0, False)


@pytest.mark.parametrize("dtype,offset", [("f32", 1), ("bf16", 1), ("bf16", 3), ("f32", 2), ("bf16", 4)])
def test_alignment(dtype, offset):
    x, ids, m, _ = _case(300, 64, 4, dtype, seed=5)
    close(run(x, ids, "softmax", m, offset=offset), O.balance_loss(x, ids, "softmax", m), 1.0, dtype == "bf16")


@pytest.mark.parametrize("at_x,at_dx", [(8, 8), (9, 9), (9, 8), (8, 11)])
@pytest.mark.parametrize("N,E,segments", [(1, 1, False), (1, 2, False), (3, 63, False), (301, 60, False), (301, 63, True),
                                          (65, 1, False), (6001, 21, False), (5003, 257, True), (5003, 511, False),
                                          (40, 1023, True), (40, 1024, False)])
def test_bf16_rows_that_share_words_with_their_neighbours(N, E, segments, at_x, at_dx):
    """Rows that start and end inside 4-byte words, the logits inside a buffer of NaN, their gradient inside one that
    keeps its other elements."""
    lens = [N // 3, 0, N - N // 3] if segments else None
    x, ids, m, cu = _case(N, E, min(E, 3), "bf16", seed=N + E, lens=lens, mask=N > 1)
    flat = torch.full((N * E + 32,), float("nan"), dtype=torch.bfloat16, device="cuda")
    out = torch.full((N * E + 32,), 7.0, dtype=torch.bfloat16, device="cuda")
    xd, dx = flat[at_x:at_x + N * E].view(N, E), out[at_dx:at_dx + N * E].view(N, E)
    xd.copy_(x)
    B = len(lens) if segments else 1
    idd, md = torch.from_numpy(ids).cuda(), None if m is None else torch.from_numpy(m).cuda()
    cud = None if cu is None else torch.from_numpy(cu).cuda()
    loss, sums, one = torch.empty(1, device="cuda"), torch.empty(B, E, device="cuda"), torch.ones(1, device="cuda")
    counts, rows = torch.empty(B, E, dtype=torch.int64, device="cuda"), torch.empty(B, dtype=torch.int64, device="cuda")
    ws = sao.balance_workspace(N, E, B)
    sao.sao_balance_loss_fwd(xd, idd, 0, loss, counts, sums, rows, ws, row_mask=md, cu_seqlens=cud)
    sao.sao_balance_loss_bwd(xd, ids.shape[1], 0, counts, rows, one, dx, ws, row_mask=md, cu_seqlens=cud)
    got = {"loss": loss.item(), "counts": counts.cpu().numpy(), "sums": sums.double().cpu().numpy(),
           "rows": rows.cpu().numpy(), "dlogits": dx.double().cpu().numpy()}
    close(got, O.balance_loss(x, ids, "softmax", m, cu), 1.0, True)
    assert (out[:at_dx] == 7).all() and (out[at_dx + N * E:] == 7).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [12, 128])
def test_masked_rows_dropped_choices_and_extreme_logits(E, score):
    x, ids, m, _ = _case(200, E, 3, seed=6)
    m[:8] = 1
    m[8:11] = 0
    ids[0] = -1
    ids[1, 1] = -2 ** 31
    x[2] = -float("inf")                       # a row that may go nowhere
    x[3] = torch.finfo(torch.float32).min      # the type's lowest value everywhere
    x[4, 1:] = torch.finfo(torch.float32).min
    x[5, :5] = -float("inf")
    x[6] = 1e30
    x[7] = -90.0
    ref = O.balance_loss(x, ids, score, m)
    x[8], x[9] = float("nan"), float("inf")    # masked
    ids[10] = 2 ** 31 - 1
    sao.sao_set_checked(True)
    try:
        got = run(x, ids, score, m)
    finally:
        sao.sao_set_checked(False)
    close(got, ref, 1.0, False)
    assert (got["dlogits"][8:11] == 0).all()


def test_nothing_counted():
    x, ids, m, cu = _case(90, 16, 2, seed=7, lens=[40, 0, 50])
    m[:] = 0
    for c in (None, cu):
        got = run(x, ids, "softmax", m, c)
        assert got["loss"] == 0 and (got["counts"] == 0).all() and (got["sums"] == 0).all()
        assert (got["rows"] == 0).all() and (got["dlogits"] == 0).all()
    e = torch.zeros(0, 16)
    got = run(e, np.zeros((0, 2), np.int32), "softmax")
    assert got["loss"] == 0 and got["rows"].tolist() == [0]


def test_device_checks():
    x, ids, m, cu = _case(90, 16, 2, seed=8, lens=[40, 0, 50])
    want = O.balance_loss(x, ids, "softmax", None)
    sao.sao_set_checked(True)
    try:
        bad = ids.copy()
        bad[3, 1] = 16
        with pytest.raises(sao.SaoError, match="expert-id"):
            run(x, bad, "softmax")
        for broken in ([0, 40, 39, 90], [1, 40, 40, 90], [0, 40, 40, 89]):
            with pytest.raises(sao.SaoError, match="cu_seqlens"):
                run(x, ids, "softmax", None, np.array(broken, np.int32), fwd_only=True)
        close(run(x, ids, "softmax"), want, 1.0, False)
    finally:
        sao.sao_set_checked(False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,E,k", [(37, 4, 4), (300, 12, 12), (500, 8, 1)])
def test_an_even_load_has_no_gradient(N, E, k, score):
    x, ids, _, _ = _case(N, E, k, seed=N, mask=False)
    if k == 1:
        ids = (np.arange(N, dtype=np.int32) % E)[:N // E * E, None].copy()
        x = x[:N // E * E]
    got = run(x, ids, score)
    assert (got["dlogits"] == 0).all() and abs(got["loss"] - 1) <= (16 + 4 * np.sqrt(N)) * U


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient_against_differences(score):
    """Central differences of the kernels' loss along random directions of at most 1 an element: the curvature term
    is below d^2 |loss| and the loss's rounding (40 u) enters over d."""
    x, ids, m, cu = _case(400, 24, 3, seed=9, lens=[100, 1, 0, 299])
    got = run(x, ids, score, m, cu)
    D = torch.rand(x.shape, generator=torch.Generator().manual_seed(10)) * 2 - 1
    d = 0.02
    up, down = run(x + d * D, ids, score, m, cu)["loss"], run(x - d * D, ids, score, m, cu)["loss"]
    slope = (got["dlogits"] * D.double().numpy()).sum()
    assert abs((up - down) / (2 * d) - slope) <= (d * d + 40 * U / d) * got["loss"]


def test_ranks_that_balance_their_joint_batch():
    """Counts, sums and rows of two halves added up give the whole batch's loss and gradient."""
    x, ids, m, _ = _case(300, 32, 4, seed=11)
    ref = O.balance_loss(x, ids, "softmax", m)
    parts, state = [], []
    for sl in (slice(0, 120), slice(120, 300)):
        xd, idd, md = x[sl].cuda(), torch.from_numpy(ids[sl]).cuda(), torch.from_numpy(m[sl]).cuda()
        loss, sums = torch.empty(1, device="cuda"), torch.empty(1, 32, device="cuda")
        counts, rows = torch.empty(1, 32, dtype=torch.int64, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
        ws = sao.balance_workspace(len(xd), 32)
        sao.sao_balance_loss_fwd(xd, idd, 0, loss, counts, sums, rows, ws, row_mask=md)
        parts.append((counts, sums, rows))
        state.append((xd, md, ws))
    counts, sums, rows = (a + b for a, b in zip(*parts))
    loss = 32 / (4 * rows.item() ** 2) * float((counts.double() * sums.double()).sum())
    assert loss == pytest.approx(ref["loss"], rel=1e-5)
    got = []
    for xd, md, ws in state:
        dx = torch.empty_like(xd)
        sao.sao_balance_loss_bwd(xd, 4, 0, counts, rows, torch.ones(1, device="cuda"), dx, ws, row_mask=md)
        got.append(dx.double().cpu().numpy())
    tol = 32 * U * ref["s"] * np.abs(ref["w"]).max(1, keepdims=True)
    assert (np.abs(np.concatenate(got) - ref["dlogits"]) <= tol + 1e-37).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_on_any_stream_and_in_a_graph(dtype):
    lens = [900, 0, 5000, 17, 40000]
    x, ids, m, cu = _case(sum(lens), 48, 4, dtype, seed=12, lens=lens)
    first = run(x, ids, "softmax", m, cu)
    again = run(x, ids, "softmax", m, cu, stream=torch.cuda.Stream())
    for k in first:
        assert np.array_equal(first[k], again[k]), k
    xd, idd, md, cud = x.cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(m).cuda(), torch.from_numpy(cu).cuda()
    B, E = len(lens), 48
    loss, sums, dx = torch.empty(1, device="cuda"), torch.empty(B, E, device="cuda"), torch.empty_like(xd)
    counts, rows = torch.empty(B, E, dtype=torch.int64, device="cuda"), torch.empty(B, dtype=torch.int64, device="cuda")
    one, ws = torch.ones(1, device="cuda"), sao.balance_workspace(len(x), E, B)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sao.sao_balance_loss_fwd(xd, idd, 0, loss, counts, sums, rows, ws, row_mask=md, cu_seqlens=cud)
        sao.sao_balance_loss_bwd(xd, 4, 0, counts, rows, one, dx, ws, row_mask=md, cu_seqlens=cud)
    for _ in range(2):
        dx.fill_(float("nan"))
        loss.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert loss.item() == first["loss"] and np.array_equal(dx.double().cpu().numpy(), first["dlogits"])


def test_logits_past_32_bit_offsets():
    N, E = (1 << 21) + 77, 1024
    x = torch.zeros(N, E, dtype=torch.bfloat16, device="cuda")
    x[-1, 5] = 3.0
    ids = torch.full((N, 1), 5, dtype=torch.int32, device="cuda")
    ids[:-1] = torch.arange(N - 1, device="cuda", dtype=torch.int32)[:, None] % E
    loss, sums, dx = torch.empty(1, device="cuda"), torch.empty(1, E, device="cuda"), torch.empty_like(x)
    counts, rows = torch.empty(1, E, dtype=torch.int64, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
    ws = sao.balance_workspace(N, E)
    sao.sao_balance_loss_fwd(x, ids, 0, loss, counts, sums, rows, ws)
    assert rows.item() == N and int(counts.sum()) == N and loss.item() == pytest.approx(1.0, rel=1e-4)
    assert torch.equal(counts[0], torch.bincount(ids[:, 0].long(), minlength=E))
    g = torch.full((1,), 1e6, device="cuda")
    sao.sao_balance_loss_bwd(x, 1, 0, counts, rows, g, dx, ws)
    w = 1e6 * E * counts[0].double() / float(N) ** 2
    for t in (0, N - 2, N - 1):
        s = torch.softmax(x[t].double(), 0)
        d = s * (w - (s * w).sum())
        assert (dx[t].double() - d).abs().max() <= 2.0 ** -8 * d.abs().max() + 32 * U * float(s.max() * w.max())
