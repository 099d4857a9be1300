"""Distillation from a teacher's top logits against fp64.

Bounds, with u = 2^-24 and S the largest sum_k |H_tk W_vk| / T. A logit of a bf16
head: products exact, sums of up to 512 elements truncated 32 times, each time by up to
2u of a partial sum that is half of the whole on average, the parts added in fp32:
(32 + h / 256) u S. Of an fp32 head (see
test_gpu_logprobs_f32.py): (8 + h / 32) u S. Both get the exponentials' and
merges' share, 16 u (1 + |lse|); the loss is a weighted mean of differences of
two such values, and its teacher's terms add 16 u (1 + |la|). Gradients in the
2-norm: a bf16 head rounds dZ once (2^-9) and bf16 outputs again (2^-9), random
signs, so 2^-7 leaves a factor of two over their sum and 2^-8 one over dZ's alone
(fp32 dW); an fp32 head as the log-probs', 1e-5."""
import numpy as np
import pytest
import torch

from oracle import sao_oracle as O
from paper_2607_07508_gb300 import sao

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(N, h, V, K, dtype="bf16", top="f32", seed=0, scale=0.05, rest=True, fill=True):
    g = torch.Generator().manual_seed(seed)
    r = np.random.Generator(np.random.PCG64(seed))
    H = torch.randn(N, h, generator=g).to(DT[dtype])
    W = (torch.randn(V, h, generator=g) * scale).to(DT[dtype])
    ids = np.stack([r.permutation(V)[:K] for _ in range(N)]).astype(np.int32) if V <= 50000 else None
    a = (torch.randn(N, K, generator=g) * 2).to(DT[top])
    if fill and K > 1:  # a third of the rows have fewer entries, anywhere in the row
        few = r.random(N) < 0.33
        ids[few[:, None] & (r.random((N, K)) < 0.5)] = -1
    c = dict(H=H, W=W, ids=ids, a=a, T=1.0, lse=None, mask=None, G=r.normal(size=N).astype(np.float32))
    c["G"][r.random(N) < 0.2] = 0
    if N == 1:
        c["G"][:] = 0.7
    if rest:
        with_rest(c, r)
    return c


def with_rest(c, r):
    a = np.where(c["ids"] >= 0, c["a"].double().numpy() / c["T"], -np.inf)
    top = np.maximum(a.max(1), -50.0)
    s = np.exp(a - top[:, None]).sum(1)
    c["lse"] = (top + np.log(np.maximum(s, 1e-20)) + r.uniform(0.01, 1.0, len(s))).astype(np.float32)


def run(c, dw="same", prev=None, stream=None, bwd=True):
    H, W = c["H"].cuda(), c["W"].cuda()
    N, h = H.shape
    V, K = W.shape[0], c["ids"].shape[1]
    ids, a = torch.from_numpy(c["ids"]).cuda(), c["a"].cuda()
    tl = None if c["lse"] is None else torch.from_numpy(c["lse"]).cuda()
    m = None if c["mask"] is None else torch.from_numpy(c["mask"]).cuda()
    nan = float("nan")
    o = {k: torch.full((N,), nan, device="cuda") for k in ("loss", "lse", "lse_rest")}
    o["z_top"] = torch.full((N, K), nan, device="cuda")
    ws = sao.distill_workspace(N, h, V, K, H.dtype)
    ws.fill_(255)
    torch.cuda.synchronize()  # `stream` does not wait for the one that the inputs were made on
    sao.sao_distill_loss_fwd(H, W, ids, a, c["T"], o["loss"], o["lse"], o["lse_rest"], o["z_top"], ws, teacher_lse=tl,
                             row_mask=m, stream=stream)
    if bwd:
        G = torch.from_numpy(c["G"]).cuda()
        o["dH"] = torch.full_like(H, nan)
        o["dW"] = (torch.full((V, h), nan, device="cuda", dtype=H.dtype if dw == "same" else DT[dw]) if prev is None
                   else prev.clone().cuda())
        torch.cuda.synchronize()
        ws.fill_(255)
        torch.cuda.synchronize()
        sao.sao_distill_loss_bwd(H, W, ids, a, c["T"], o["lse"], o["lse_rest"], o["z_top"],
                                 G, o["dH"], o["dW"], ws, teacher_lse=tl,
                                 accumulate_dW=prev is not None, stream=stream)
    torch.cuda.synchronize()
    return {k: v.double().cpu().numpy() for k, v in o.items()}


def want(c):
    return O.distill_loss(c["H"], c["W"], c["ids"], c["a"], c["T"], c["lse"], c["mask"],
                          np.where(c["mask"] == 0, 0, c["G"]) if c["mask"] is not None else c["G"])


def bound(c):
    H, W = np.abs(c["H"].double().numpy()), np.abs(c["W"].double().numpy())
    H = np.where(np.isfinite(H), H, 0)
    h = H.shape[1]
    S = (H @ W.T).max() / c["T"]
    return ((32 + h / 256) if c["H"].dtype == torch.bfloat16 else (8 + h / 32)) * U * S


def close(got, ref, c, grads=True, dw_tol=None):
    z = bound(c)
    fin = np.isfinite(ref["loss"])
    assert np.array_equal(np.isfinite(got["loss"]), fin)
    ok = lambda g, w, tol: np.abs(g - w).max(initial=0.0) <= tol
    e = 16 * U * (1 + np.abs(ref["lse"]).max())
    assert ok(got["lse"], ref["lse"], z + e)
    la = 0.0 if c["lse"] is None else np.abs(c["lse"][np.isfinite(c["lse"])]).max(initial=0.0)
    a = np.abs(c["a"].double().numpy())
    a = a[a < 1e30].max(initial=0.0) / c["T"]
    assert ok(got["loss"][fin], ref["loss"][fin], 2 * (z + e) + 16 * U * (1 + la + a))
    assert np.array_equal(np.isnan(got["lse_rest"]), np.isnan(ref["lse_rest"]))
    r = np.isfinite(ref["lse_rest"])
    assert np.array_equal(got["lse_rest"] == -np.inf, ref["lse_rest"] == -np.inf)
    assert ok(got["lse_rest"][r], ref["lse_rest"][r], z + 16 * U * (1 + np.abs(ref["lse_rest"][r]).max(initial=0.0)))
    if grads:
        bf = c["H"].dtype == torch.bfloat16
        for k, tol in (("dH", 2.0 ** -7 if bf else 1e-5), ("dW", dw_tol or (2.0 ** -7 if bf else 1e-5))):
            assert np.isfinite(got[k]).all(), k
            n = np.linalg.norm(ref[k])
            assert np.linalg.norm(got[k] - ref[k]) <= tol * n + 1e-30, (k, np.linalg.norm(got[k] - ref[k]) / max(n, 1e-300))


SIZES = [(1, 8, 1, 1), (1, 64, 300, 5), (2, 16, 257, 256), (127, 72, 257, 17), (128, 256, 512, 1), (129, 64, 5000, 64),
         (300, 520, 1000, 33), (65, 1032, 3001, 100), (31, 2048, 2000, 20)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("N,h,V,K", SIZES)
def test_against_fp64(N, h, V, K, rest, dtype):
    c = _case(N, h + (0 if dtype == "bf16" else 3), V, K, dtype, top="f32" if N % 2 else "bf16", seed=N + K, rest=rest)
    if N == 129:
        c["T"] = 2.0
        if rest:
            with_rest(c, np.random.Generator(np.random.PCG64(1)))
    if N >= 127:
        c["mask"] = (np.random.Generator(np.random.PCG64(2)).random(N) < 0.7).astype(np.uint8)
        c["G"] *= c["mask"]
    ref = want(c)
    got = run(c)
    close(got, ref, c)
    valid = c["ids"] >= 0
    if c["mask"] is not None:
        valid &= c["mask"][:, None] != 0
        assert (got["loss"][c["mask"] == 0] == 0).all() and (got["dH"][c["mask"] == 0] == 0).all()
    assert np.abs(got["z_top"] - np.where(valid, ref["z_top"], 0)).max() <= bound(c) + 2 * U * np.abs(ref["z_top"]).max()


@pytest.mark.parametrize("N,h,V,K", [(1, 8, 9, 4), (1, 2048, 5003, 20), (1, 2056, 700, 33), (1, 6144, 900, 7), (1, 6152, 900, 7),
                                     (2, 1000, 2500, 300), (2, 4096, 311, 64), (3, 2048, 2000, 50), (4, 520, 80000, 1024),
                                     (4, 2056, 300, 12), (2, 16, 400000, 100)])
def test_few_rows(N, h, V, K):
    """One or two rows of a bf16 head go through W in one pass: sums in fp32 throughout, dZ unrounded."""
    for rest in (False, True):
        g = torch.Generator().manual_seed(h)
        c = _case(N, h, min(V, 50000), K, seed=V, rest=False, scale=0.02)
        c["W"] = (torch.randn(V, h, generator=g) * 0.02).bfloat16()
        r = np.random.Generator(np.random.PCG64(V))
        ids = np.stack([r.permutation(V)[:K] for _ in range(N)]).astype(np.int32)
        c["ids"] = np.where(c["ids"] >= 0, ids, -1).astype(np.int32)
        if rest:
            with_rest(c, r)
        c["G"] = r.normal(size=N).astype(np.float32)
        if N > 1:
            c["mask"] = np.ones(N, np.uint8)
            c["mask"][1], c["G"][1] = 0, 0
            c["H"][1] = float("nan")
        else:
            c["T"] = 0.7
            if rest:
                with_rest(c, r)
        clean = {**c, "H": torch.nan_to_num(c["H"])}
        ref = want(clean)
        close(run(c), ref, clean)
        if h * V < 1 << 23:
            close(run(c, dw="f32"), ref, clean, dw_tol=1e-5 if h <= (6144 if N == 1 else 2048 if N == 2 else 0) else 2.0 ** -8)
            prev = torch.randn(V, h) * 0.01
            got = run(c, prev=prev)
            assert np.linalg.norm(got["dW"] - prev.double().numpy() - ref["dW"]) <= 2.0 ** -8 * np.linalg.norm(ref["dW"])


@pytest.mark.parametrize("N,h,V,K", [(1, 1, 9, 4), (1, 256, 4096, 8), (1, 515, 3001, 20), (1, 1024, 5003, 33), (1, 1025, 700, 5),
                                     (1, 2048, 900, 7), (1, 2052, 900, 7), (1, 4096, 313, 64), (1, 4095, 313, 64),
                                     (1, 4100, 300, 12), (2, 96, 2500, 300), (3, 1024, 20000, 1024), (4, 1023, 700, 11),
                                     (4, 2047, 300, 9), (4, 2048, 500, 50), (5, 2048, 300, 9), (5, 40, 40000, 100),
                                     (7, 515, 1000, 64), (8, 1024, 2000, 20), (8, 1022, 311, 3), (9, 1024, 700, 20)])
def test_few_rows_of_an_fp32_head(N, h, V, K):
    for rest in (False, True):
        c = _case(N, h, V, K, "f32", seed=V + h, rest=False, scale=0.03)
        r = np.random.Generator(np.random.PCG64(V))
        c["T"] = 0.7 if N == 1 else 2.0
        if rest:
            with_rest(c, r)
        c["G"] = r.normal(size=N).astype(np.float32)
        if N > 1:
            c["mask"] = np.ones(N, np.uint8)
            c["mask"][1], c["G"][1] = 0, 0
            c["H"][1] = float("nan")
        clean = {**c, "H": torch.nan_to_num(c["H"])}
        ref = want(clean)
        close(run(c), ref, clean)
        prev = torch.randn(V, h) * 0.01
        got = run(c, prev=prev)
        d = got["dW"] - prev.double().numpy() - ref["dW"]
        assert np.linalg.norm(d) <= 1e-5 * np.linalg.norm(ref["dW"]) + 2 * U * np.linalg.norm(prev.double().numpy())


@pytest.mark.parametrize("at", [1, 2, 4])
def test_few_rows_inside_a_buffer(at):
    """fp32 operands off 16-byte alignment, between elements that are not theirs."""
    N, h, V, K = 3, 256, 700, 9
    c = _case(N, h, V, K, "f32", seed=at, rest=False)
    c["G"][:] = [0.5, -1.0, 2.0]
    ref = want(c)

    def inside(x, fill):
        flat = torch.full((x.numel() + 8,), fill, device="cuda")
        flat[at:at + x.numel()] = x.flatten().cuda()
        return flat, flat[at:at + x.numel()].view(x.shape)

    H, W = inside(c["H"], float("nan"))[1], inside(c["W"], float("nan"))[1]
    (dh_buf, dH), (dw_buf, dW) = inside(torch.zeros(N, h), 7.0), inside(torch.zeros(V, h), 7.0)
    ids, a, G = torch.from_numpy(c["ids"]).cuda(), c["a"].cuda(), torch.from_numpy(c["G"]).cuda()
    o = {k: torch.empty(N, device="cuda") for k in ("loss", "lse", "lse_rest")}
    z = torch.empty(N, K, device="cuda")
    ws = sao.distill_workspace(N, h, V, K, torch.float32)
    sao.sao_distill_loss_fwd(H, W, ids, a, 1.0, o["loss"], o["lse"], o["lse_rest"], z, ws)
    sao.sao_distill_loss_bwd(H, W, ids, a, 1.0, o["lse"], o["lse_rest"], z, G, dH, dW, ws)
    close({k: v.double().cpu().numpy() for k, v in {**o, "dH": dH, "dW": dW}.items()}, ref, c)
    for buf, n in ((dh_buf, N * h), (dw_buf, V * h)):
        assert (buf[:at] == 7).all() and (buf[at + n:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,K", [(5, 5), (256, 256), (300, 300), (1100, 1024)])
def test_entries_that_fill_tiles_or_the_vocabulary(V, K, dtype):
    """Whole tiles (and quarter tiles) without a column of the rest, and no rest at all."""
    for rest in (False, True):
        c = _case(70, 48, V, K, dtype, seed=V, rest=rest, fill=False)
        if V == 1100:
            c["ids"] = np.tile(np.arange(K, dtype=np.int32)[::-1], (70, 1)).copy()
        close(run(c), want(c), c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_entries_in_one_tile(dtype):
    c = _case(200, 64, 4000, 250, dtype, seed=3)
    r = np.random.Generator(np.random.PCG64(3))
    c["ids"] = np.stack([1024 + r.permutation(256)[:250] for _ in range(200)]).astype(np.int32)
    close(run(c), want(c), c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_student_with_all_its_mass_on_the_entries(dtype):
    """q_rest down to e^-30: lse_rest and the divergence's last term keep their digits, nothing overflows."""
    c = _case(64, 64, 700, 3, dtype, seed=4, fill=False)
    W = c["W"].float()
    for t in range(64):
        c["H"][t] = (W[c["ids"][t, 0]] * (30.0 * (t + 1) / 64 / float(W[c["ids"][t, 0]].square().sum()))).to(c["H"].dtype)
    ref = want(c)
    assert np.nanmin(ref["lse_rest"] - ref["lse"]) < -15
    close(run(c), ref, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
def test_rows_without_a_teacher_and_wrong_rows(dtype, rest):
    c = _case(140, 40, 900, 6, dtype, seed=5, rest=rest, fill=False)
    c["G"][:] = 1.0
    c["ids"][0] = -1                        # no entry
    c["ids"][1] = -7                        # any negative id
    c["a"][2] = -float("inf")               # no finite logit
    c["ids"][3, 1] = c["ids"][3, 4]         # one id twice
    c["ids"][4, 5] = 900                    # out of range
    c["ids"][5, 0] = 2 ** 31 - 1
    c["a"][6, 2] = float("nan")
    c["a"][7, 2] = float("inf")
    c["a"][8, 2] = -float("inf")            # one entry that the teacher never picks
    c["a"][9, 1] = torch.finfo(torch.float32).min
    if rest:
        c["lse"][10] = np.nan
        c["lse"][11] = -2000.0              # not a log-sum-exp of these logits: exp overflows
    ref = want(c)
    got = run(c)
    close(got, ref, c)
    none = np.isnan(ref["lse_rest"])
    assert {3, 4, 5, 6, 7} <= set(np.flatnonzero(none)) and (got["dH"][none] == 0).all()
    assert (got["loss"][:2] == 0).all() or rest
    sao.sao_set_checked(True)
    try:
        with pytest.raises(sao.SaoError, match="teacher-entry"):
            run(c, bwd=False)
        for row in (3, 4, 5):
            c["ids"][row] = np.arange(6)
        run(c, bwd=False)
    finally:
        sao.sao_set_checked(False)


@pytest.mark.parametrize("N", [40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_rows_may_hold_anything(N, dtype):
    c = _case(N, 72, 30000, 9, dtype, seed=6)
    c["mask"] = (np.arange(N) % 3 != 1).astype(np.uint8)
    off = c["mask"] == 0
    c["G"][off] = 0
    clean, ref, plain = run(c), want(c), {**c, "H": c["H"].clone(), "a": c["a"].clone(), "lse": c["lse"].copy()}
    c["H"][torch.from_numpy(off)] = float("nan")
    c["a"][torch.from_numpy(off)] = float("inf")
    c["lse"][off] = np.nan
    c["ids"][off] = 2 ** 31 - 1
    sao.sao_set_checked(True)
    try:
        got = run(c)
    finally:
        sao.sao_set_checked(False)
    # an fp32 forward of few rows runs over the masked ones too: their NaN sends its products to the FMA tiles
    if dtype == "f32":
        close(got, ref, plain)
    for k in clean if dtype == "bf16" else ():
        assert np.array_equal(clean[k], got[k], equal_nan=k == "lse_rest"), k
    c["mask"][:] = 0
    c["G"][:] = 0
    got = run(c)
    assert (got["loss"] == 0).all() and (got["dH"] == 0).all() and (got["dW"] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_chunks_of_the_vocabulary(dtype):
    c = _case(700, 64, 5000, 40, dtype, seed=7)
    ref = want(c)
    whole = run(c)
    sao.sao_set_dz_budget_bytes(1 << 20)
    try:
        cut = run(c)
    finally:
        sao.sao_set_dz_budget_bytes(4 << 30)
    close(whole, ref, c)
    close(cut, ref, c)


@pytest.mark.parametrize("N", [40, 300, 1500])
def test_cta_pairs(N):
    c = _case(N, 1096, 3000, 40, "bf16", seed=15)
    c["mask"] = (np.arange(N) % 7 != 3).astype(np.uint8)
    c["G"] *= c["mask"]
    ref = want(c)
    sao.sao_set_cta_pairs(True)
    try:
        close(run(c), ref, c)
        got = run(c, dw="f32")
    finally:
        sao.sao_set_cta_pairs(False)
    close(got, ref, c, dw_tol=2.0 ** -8)


@pytest.mark.parametrize("N", [90, 1500, 4000])
def test_bf16_head_with_an_fp32_dW(N):
    c = _case(N, 136, 700, 11, "bf16", seed=8)
    ref = want(c)
    close(run(c, dw="f32"), ref, c, dw_tol=2.0 ** -8)
    prev = torch.randn(700, 136) * 0.1
    got = run(c, prev=prev)
    assert np.linalg.norm(got["dW"] - prev.double().numpy() - ref["dW"]) <= 2.0 ** -8 * np.linalg.norm(ref["dW"])


@pytest.mark.parametrize("N,K,ties", [(65, 1, False), (130, 1, False), (130, 3, True), (700, 1, False), (5000, 2, False),
                                      (8192, 1, True)])
def test_rows_that_dominate_keep_their_entries(N, K, ties):
    """A few rows carry most of the gradient, with entries half way between two bf16 values. Theirs are kept to
    2^-16, the other rows' to 2^-8 of a tenth; a bf16 output adds at most 2^-8 / sqrt(3) in the 2-norm."""
    c = _case(N, 64, 2000, K, seed=N, rest=False, fill=False)
    c["a"][:, 1:] = -60.0
    r = np.random.Generator(np.random.PCG64(N))
    heavy = r.permutation(N)[:5]
    c["G"] = (r.uniform(0.5, 1, N) * 0.2 / np.sqrt(N)).astype(np.float32)
    if ties:
        c["G"][:] = np.float32(0.2 / np.sqrt(N) * (1 + 2.0 ** -8))
    c["G"][heavy] = 1 + 2.0 ** -8
    ref = want(c)
    got = run(c, dw="f32")
    close(got, ref, c)
    err = lambda k: np.linalg.norm(got[k] - ref[k]) / np.linalg.norm(ref[k])
    assert err("dW") <= 2.0 ** -8 * 0.11
    assert err("dH") <= 2.0 ** -8 / np.sqrt(3) + 2.0 ** -11
    got = run(c)
    assert max(err("dW"), err("dH")) <= 2.0 ** -8 / np.sqrt(3) + 2.0 ** -11
    again = run(c)
    assert all(np.array_equal(got[k], again[k]) for k in ("dH", "dW"))


def test_fp32_dW_is_added_to():
    c = _case(130, 61, 700, 11, "f32", seed=9)
    ref = want(c)
    prev = torch.randn(700, 61)
    got = run(c, prev=prev)
    both = np.linalg.norm(ref["dW"]) + np.linalg.norm(prev.numpy())
    assert np.linalg.norm(got["dW"] - prev.double().numpy() - ref["dW"]) <= 1e-5 * both


def test_operands_outside_the_splitting():
    """fp32 operands of 2^70 and 2^-70 take fp32 FMA tiles, entries and all."""
    c = _case(150, 40, 1000, 30, "f32", seed=10)
    plain = want(c)
    c["H"] *= 2.0 ** 70
    c["W"] *= 2.0 ** -70
    got = run(c)
    got["dH"], plain["dH"] = got["dH"] * 2.0 ** 70, plain["dH"]
    got["dW"] = got["dW"] * 2.0 ** -70
    c["H"] *= 2.0 ** -70
    c["W"] *= 2.0 ** 70
    close(got, plain, c)


@pytest.mark.parametrize("rest", [False, True])
def test_gradient_against_differences(rest):
    """Central differences of the kernels' own fp32 losses along random directions. With a step of d the
    difference's curvature term is below d^2 times the third derivative (at most |direction logit|^3), and the
    losses' rounding enters as err / d: for |direction logits| <= 1 and err below 1e-5 a row, d = 0.05 leaves
    2.5e-3 + 2e-4 a row."""
    c = _case(60, 32, 400, 12, "f32", seed=11, rest=rest, scale=0.3)
    c["T"] = 1.5
    if rest:
        with_rest(c, np.random.Generator(np.random.PCG64(5)))
    got = run(c)
    g = torch.Generator().manual_seed(12)
    d, G = 0.05, c["G"].astype(np.float64)
    H, W = c["H"].clone(), c["W"].clone()
    for which in ("H", "W"):
        D = torch.randn(c[which].shape, generator=g)
        other = W if which == "H" else H
        D /= (D @ other.t()).abs().max() / c["T"]
        loss = []
        for sign in (1, -1):
            c["H"], c["W"] = H.clone(), W.clone()
            c[which] += sign * d * D
            loss.append((G * run(c, bwd=False)["loss"]).sum())
        slope = (got["d" + which] * D.double().numpy()).sum()
        assert abs((loss[0] - loss[1]) / (2 * d) - slope) <= np.abs(G).sum() * 2.7e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_on_any_stream_and_in_a_graph(dtype):
    c = _case(517, 256, 9000, 20, dtype, seed=13)
    first = run(c)
    again = run(c, stream=torch.cuda.Stream())
    for k in first:
        assert np.array_equal(first[k], again[k], equal_nan=True), k
    dev = {k: (v.cuda() if torch.is_tensor(v) else torch.from_numpy(v).cuda()) for k, v in c.items()
           if k in ("H", "W", "ids", "a", "lse", "G")}
    N, K = c["ids"].shape
    o = {k: torch.empty(N, device="cuda") for k in ("loss", "lse", "lse_rest")}
    o["z_top"] = torch.empty(N, K, device="cuda")
    o["dH"], o["dW"] = torch.empty_like(dev["H"]), torch.empty_like(dev["W"])
    ws = sao.distill_workspace(N, 256, 9000, K, dev["H"].dtype)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sao.sao_distill_loss_fwd(dev["H"], dev["W"], dev["ids"], dev["a"], 1.0, o["loss"], o["lse"], o["lse_rest"],
                                 o["z_top"], ws, teacher_lse=dev["lse"])
        sao.sao_distill_loss_bwd(dev["H"], dev["W"], dev["ids"], dev["a"], 1.0, o["lse"], o["lse_rest"], o["z_top"],
                                 dev["G"], o["dH"], o["dW"], ws, teacher_lse=dev["lse"])
    for v in o.values():
        v.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    for k in first:
        assert np.array_equal(first[k], o[k].double().cpu().numpy(), equal_nan=True), k


def test_entries_past_32_bit_offsets():
    """2^31 entries and more: the last rows against fp64, all else in place."""
    N, h, V, K = (1 << 21) + 130, 8, 1200, 1024
    g = torch.Generator(device="cuda").manual_seed(14)
    H = torch.randn(N, h, generator=g, device="cuda").bfloat16()
    W = (torch.randn(V, h, generator=g, device="cuda") * 0.3).bfloat16()
    ids = (torch.arange(K, device="cuda", dtype=torch.int32)[None] * 7 + torch.arange(N, device="cuda", dtype=torch.int32)[:, None] % 97) % V
    ids = ids.contiguous()
    a = torch.randn(K, generator=g, device="cuda").repeat(N, 1).bfloat16()
    G = torch.zeros(N, device="cuda")
    G[-3:] = 1.0
    G[5] = 1.0
    o = {k: torch.empty(N, device="cuda") for k in ("loss", "lse", "lse_rest")}
    z_top = torch.empty(N, K, device="cuda")
    ws = sao.distill_workspace(N, h, V, K)
    dH, dW = torch.empty_like(H), torch.empty(V, h, device="cuda")
    sao.sao_distill_loss_fwd(H, W, ids, a, 1.0, o["loss"], o["lse"], o["lse_rest"], z_top, ws)
    sao.sao_distill_loss_bwd(H, W, ids, a, 1.0, o["lse"], o["lse_rest"], z_top, G, dH, dW, ws)
    rows = torch.tensor([5, N - 3, N - 2, N - 1], device="cuda")
    c = dict(H=H[rows].cpu(), W=W.cpu(), ids=ids[rows].cpu().numpy(), a=a[rows].cpu(), T=1.0, lse=None, mask=None,
             G=np.ones(4, np.float32))
    ref = want(c)
    got = {k: v[rows].double().cpu().numpy() for k, v in o.items()}
    got.update(dH=dH[rows].double().cpu().numpy(), dW=dW.double().cpu().numpy())
    close(got, ref, c, dw_tol=2.0 ** -8)
    assert int((dH != 0).any(1).sum()) == 4 and bool(torch.isfinite(o["loss"]).all())
