"""The feed-forward operators in workspaces of exactly the size asked for, between guard bytes: right results, and nothing written beside
them, whatever offsets and pairs hold."""
import ctypes

import numpy as np
import pytest
import torch

from test_moe_experts_gpu import Case, dev, order

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

GUARD = 1 << 16


class Guarded:
    """A workspace of n bytes (its counters zero, the rest NaN) and GUARD bytes on either side of it."""

    def __init__(self, n):
        self.buf = torch.full((2 * GUARD + n,), 0xA5, dtype=torch.uint8, device="cuda")
        self.ws = self.buf[GUARD:GUARD + n]
        self.ws.fill_(0xFF)
        self.ws[:65536].zero_()

    def check(self, what):
        torch.cuda.synchronize()
        n = self.ws.numel()
        assert (self.buf[:GUARD] == 0xA5).all() and (self.buf[GUARD + n:] == 0xA5).all(), what


def experts_bytes(c):
    s = nmm.nmm_moe_ffn(tokens=c.T, top_k=c.k, experts=c.E, first=c.first, local=c.local, hidden=c.hidden, inner=c.inner)
    return nmm.lib().nmm_moe_experts_workspace_size(ctypes.byref(s))


@pytest.mark.parametrize("T,E,k,hidden,inner", [(1, 8, 8, 96, 48), (6, 8, 4, 88, 40), (14, 16, 4, 97, 49), (40, 64, 8, 520, 260),
                                                (64, 8, 4, 96, 48), (130, 3, 2, 1037, 531), (300, 2, 1, 1032, 520), (3, 6, 2, 4096, 70)])
def test_experts_whatever_the_indices_hold(T, E, k, hidden, inner):
    rng = np.random.default_rng(T)
    c = Case(T, T, E, k, hidden, inner, integer=True, residual=T % 2 == 0)
    g = Guarded(experts_bytes(c))
    c.check(1, workspace=g.ws)
    g.check("a choice")
    good = [t.clone() for t in c.route]
    P, i32 = T * k, lambda a: dev(np.asarray(a, dtype=np.int64).astype(np.int32))
    bad_pairs = {"far": np.full(P, 1 << 30), "negative": np.full(P, -1), "one behind": np.full(P, P), "the same": np.zeros(P),
                 "any": rng.integers(-(1 << 31), 1 << 31, P), "reversed": good[3].cpu().numpy()[::-1]}
    for what, a in bad_pairs.items():
        c.route[3] = i32(a)
        c.run(1, workspace=g.ws)
        g.check(("pairs", what))
        assert (c.out[:, hidden:] == 7).all()
    c.route[3] = good[3]
    bad_offsets = {"all claim every pair": np.arange(E + 1) % 2 * P, "least": np.full(E + 1, -(1 << 31)), "most": np.full(E + 1, (1 << 31) - 1),
                   "least and most": np.arange(E + 1) % 2 * ((1 << 32) - 1) - (1 << 31), "descending": good[2].cpu().numpy()[::-1],
                   "one behind": good[2].cpu().numpy() + 1, "any": rng.integers(-(1 << 31), 1 << 31, E + 1),
                   "near": rng.integers(-3, P + 3, E + 1)}
    for what, a in bad_offsets.items():
        c.route[2] = i32(a)
        c.run(1, workspace=g.ws)
        g.check(("offsets", what))
        assert (c.out[:, hidden:] == 7).all()
    c.route[2] = good[2]
    c.route[0] = i32(rng.integers(-(1 << 31), 1 << 31, (T, k)))
    c.run(1, workspace=g.ws)
    g.check("chosen")
    c.route[0] = good[0]
    c.check(1, workspace=g.ws)
    g.check("a choice again")


@pytest.mark.parametrize("T,E,k", [(8, 64, 8), (64, 256, 8), (128, 1024, 8), (700, 1000, 8), (3000, 60, 6), (20000, 20, 4)])
def test_route(T, E, k):
    s = nmm.nmm_moe_router(tokens=T, experts=E, top_k=k, groups=1, top_groups=1)
    n = nmm.lib().nmm_moe_route_workspace_size(ctypes.byref(s))
    logits = torch.randn((T, E), device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    out = torch.zeros((T, k), **i32), torch.zeros((T, k), device="cuda"), torch.zeros(E + 1, **i32), torch.zeros(T * k, **i32)
    g = Guarded(n)
    for _ in range(2):
        nmm.nmm_moe_route(logits, *out, score=nmm.NMM_SCORE_SIGMOID, workspace=g.ws)
        g.check((T, E, k))
        offsets, pairs = order(out[0].cpu().numpy(), E)
        assert np.array_equal(out[2].cpu().numpy(), offsets) and np.array_equal(out[3].cpu().numpy(), pairs)
        logits.normal_()


@pytest.mark.parametrize("M,K,N,gated", [(64, 7168, 1001, True), (200, 4099, 130, False), (256, 7168, 512, True)])
def test_slices_of_a_product(M, K, N, gated):
    rows = 2 * N if gated else N
    s = nmm.nmm_nt_act(M=M, K=K, N=N, gated=gated)
    n = nmm.lib().nmm_gemv_nt_act_workspace_size(ctypes.byref(s))
    assert n > 65536
    gen = torch.Generator(device="cuda").manual_seed(M)
    ones = lambda *shape: torch.randint(-1, 2, shape, generator=gen, device="cuda").to(torch.bfloat16)
    up8 = (K + 7) // 8 * 8
    # one value in 64 of a weight's row: sums of integers that fp32 holds
    x, w = ones(M, up8), ones(rows, up8) * (torch.rand((rows, up8), generator=gen, device="cuda") < 1 / 64)
    y = torch.full((M, N + 3), 7.0, device="cuda")
    g = Guarded(n)
    nmm.nmm_gemv_nt_act(x, w, None, act=nmm.NMM_ACT_RELU, gated=gated, y_f32=y[:, :N], K=K, workspace=g.ws)
    g.check((M, K, N))
    z = x[:, :K].float() @ w[:, :K].float().T
    want = z.clamp(min=0) if not gated else z[:, :N].clamp(min=0) * z[:, N:]
    assert torch.equal(y[:, :N], want) and (y[:, N:] == 7).all()
