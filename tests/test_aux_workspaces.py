"""The auxiliary losses' workspaces: one that was sized for the largest micro-batch serves every smaller one."""
import ctypes
import random
import re

import pytest

P = ctypes.c_void_p
F32, BF16, WORKSPACE = 0, 1, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2607_07508_gb300 import build, sao
    build.build()
    return sao.load()


def _near(rng, most):
    """1 .. 300, thereabouts of the limits between the paths and of tiles, and others up to `most`, ascending."""
    n = set(range(1, 300)) | {int(2 ** rng.uniform(0, 21)) for _ in range(300)}
    for at in (64, 128, 512, 1024, 3072, 4096, 8192, 8224, 14123, 16384, 38912, 65536):
        n |= {at + d for d in (-33, -32, -31, -2, -1, 0, 1, 2, 31, 32, 33, 96, 128)}
    return sorted(k for k in n if 1 <= k <= most)


HEADS = [(2048, 151936, BF16, 20), (6144, 154880, BF16, 50), (1024, 32000, BF16, 64), (64, 151936, BF16, 3),
         (256, 4096, F32, 8), (1024, 32000, F32, 33), (515, 20000, F32, 1), (4096, 3000, F32, 1024), (40, 500, F32, 20)]


@pytest.mark.parametrize("budget", [4 << 30, 1 << 28, 1 << 20])
@pytest.mark.parametrize("h,V,dt,K", HEADS)
def test_a_distillation_of_fewer_rows_needs_no_more(lib, h, V, dt, K, budget):
    lib.sao_set_dz_budget_bytes(budget)
    try:
        last = 0
        for N in _near(random.Random(h), 1 << 21):
            size = lib.sao_distill_workspace_bytes(N, h, V, K, dt)
            assert size >= last, N
            assert lib.sao_distill_workspace_bytes(N, h, V, max(K // 2, 1), dt) <= size
            last = size
    finally:
        lib.sao_set_dz_budget_bytes(4 << 30)


def needed(lib, N, h, V, K, dt):
    """What a call says that it needs, when refused for its workspace (before anything is launched)."""
    r = lib.sao_distill_loss_fwd(P(256), P(256), dt, P(256), P(256), F32, None, None, N, h, V, K, 1.0, P(256), P(256),
                                 P(256), P(256), P(256), 256, None)
    assert r == WORKSPACE
    return int(re.search(r"(\d+) needed", lib.sao_last_error_string().decode())[1])


def _what_calls_need(lib, h, V, dt, K, budget):
    lib.sao_set_dz_budget_bytes(budget)
    try:
        for N in _near(random.Random(h + 1), 1 << 21):
            assert needed(lib, N, h, V, K, dt) <= lib.sao_distill_workspace_bytes(N, h, V, K, dt), N
    finally:
        lib.sao_set_dz_budget_bytes(4 << 30)


@pytest.mark.parametrize("budget", [4 << 30, 1 << 28, 1 << 20])
@pytest.mark.parametrize("h,V,dt,K", [c for c in HEADS if c[2] == F32])
def test_an_fp32_call_needs_no_more_than_its_workspace(lib, h, V, dt, K, budget):
    _what_calls_need(lib, h, V, dt, K, budget)


@pytest.mark.gpu  # (a bf16 head is refused without its device)
@pytest.mark.parametrize("budget", [4 << 30, 1 << 28, 1 << 20])
@pytest.mark.parametrize("h,V,dt,K", [c for c in HEADS if c[2] == BF16])
def test_a_bf16_call_needs_no_more_than_its_workspace(lib, h, V, dt, K, budget):
    _what_calls_need(lib, h, V, dt, K, budget)


def test_a_balance_of_fewer_rows_needs_no_more(lib):
    for E, B in ((8, 1), (160, 1), (63, 96), (1024, 3)):
        last = 0
        for N in _near(random.Random(E), 1 << 21):
            size = lib.sao_balance_workspace_bytes(N, E, B)
            assert size >= last, N
            assert size <= lib.sao_balance_workspace_bytes(N, E, B + 1)
            assert size <= lib.sao_balance_workspace_bytes(N, min(E + 1, 1024), B)
            last = size


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_ragged_micro_batches(dtype):
    import torch
    from paper_2607_07508_gb300 import sao
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    h, V, K = 1024, 8000, 6
    g = torch.Generator().manual_seed(1)
    W = (torch.randn(V, h, generator=g) * 0.03).to(dt).cuda()
    ws = sao.distill_workspace(8193, h, V, K, dt)
    for N in (8193, 8192, 4100, 513, 512, 129, 128, 97, 65, 64, 3, 2, 1):
        H = torch.randn(N, h, generator=g).to(dt).cuda()
        ids = (torch.arange(N, dtype=torch.int32)[:, None] * 7 + torch.arange(K, dtype=torch.int32) * 900) % V
        ids, a = ids.cuda(), torch.randn(N, K, generator=g).cuda()
        loss, lse, rest = (torch.empty(N, device="cuda") for _ in range(3))
        z, dH, dW = torch.empty(N, K, device="cuda"), torch.empty_like(H), torch.empty(V, h, device="cuda")
        sao.sao_distill_loss_fwd(H, W, ids, a, 1.0, loss, lse, rest, z, ws)
        sao.sao_distill_loss_bwd(H, W, ids, a, 1.0, lse, rest, z, torch.ones(N, device="cuda"), dH, dW, ws)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(loss).all() and torch.isfinite(dW).all() and (dH != 0).any())
