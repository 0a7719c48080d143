"""nmm_gemv_nt_act's fp32 results where K is long: one product of 2^24 among many of 3 x 2^-7.

A matrix instruction adds 32 products and what came before in at most 33 roundings of half a step, 2^-24, of the sum of magnitudes.
Results in fp32 are fp64 sums of at most four such instructions' (132 roundings), rounded once a wave or slice and added in
fp32, 16 roundings more at most: 148 in all, however long K is.  (One fp32 sum over K / 4 loses 32 x 3 x 2^-7 = 3/4 of a step of 2^24 at each
instruction behind the large product.)
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

SMALL = 3 * 2.0 ** -7
ROUNDINGS = 148


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K,N", [(1, 262144, 40), (5, 262144, 64), (16, 262143, 64), (32, 262144, 33), (50, 262144, 64), (200, 262141, 64),
                                   (1, 65536, 8200), (20, 65535, 8200), (33, 65536, 8192), (200, 65531, 8192)])
def test_a_long_sum_beside_a_large_product(M, K, N, gated, dt):
    up8 = (K + 7) // 8 * 8
    if gated:
        N //= 2
    scale = 2.0 ** (torch.arange(N, device="cuda") % 3) * (1 - 2 * (torch.arange(N, device="cuda") % 2))
    of_row = 2.0 ** -(torch.arange(M, device="cuda") % 3)
    wt = torch.zeros((2 * N if gated else N, up8), dtype=dt, device="cuda")
    x = torch.ones((M, up8), dtype=dt, device="cuda")
    wt[:N] = SMALL
    for large in (0, K // 9):
        wt[:N, large], x[:, large] = 4096.0, 4096.0
        if gated:
            wt[N:, large + 1] = 1.0                        # what the gate multiplies: x's scale
        w, xs = wt.clone(), (x * of_row[:, None]).to(dt)
        w[:N] *= scale[:, None].to(dt)
        y = torch.full((M, N + 1), 7.0, device="cuda")
        nmm.nmm_gemv_nt_act(xs, w, None, gated=gated, K=K, y_f32=y[:, :N])
        mag = (2.0 ** 24 + (K - 1) * SMALL) * of_row.double()[:, None] * scale.double()
        if gated:
            mag = mag * of_row.double()[:, None]
        off = ((y[:, :N].double() - mag) / mag).abs().max().item() * 2 ** 24
        assert off <= ROUNDINGS and (y[:, N] == 7).all(), (large, off)
        wt[:N, large], x[:, large] = SMALL, 1.0
        if gated:
            wt[N:, large + 1] = 0.0


def test_y_is_y_f32_rounded():
    for M, K, N in ((1, 704, 96), (40, 5000, 96), (140, 5000, 300)):
        x = torch.randn((M, K), device="cuda").to(torch.bfloat16)
        w = (torch.randn((N, K), device="cuda") * K ** -0.5).to(torch.bfloat16)
        y, f = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, N), device="cuda")
        nmm.nmm_gemv_nt_act(x, w, y, act=nmm.NMM_ACT_SILU, y_f32=f)
        assert torch.equal(y, f.to(torch.bfloat16))
