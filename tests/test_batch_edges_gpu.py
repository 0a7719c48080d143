"""Calls of the batched operators that their documentation allows and that lie at its edges: one query for all sequences, queries that
are not finite, more tokens than positions, plans far longer than the sequences, scales of zero and below, weights at their zero
points, every scale byte of an 8-bit row, and the cache entry beside nmm_mla_kv_update's."""
import numpy as np
import pytest
import torch

from oracle import batch as ob
from test_attention_batch_gpu import Case

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

FORMATS = pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])


@FORMATS
@pytest.mark.parametrize("H,prefix", [(16, 0), (24, 0), (70, 0), (16, 400)])
def test_one_query_for_all_sequences(H, prefix, fp8):
    c = Case(H + prefix, 5, 1, H, prefix, [70, 1, 200, 64, 33], 32, fp8)
    c.q[:] = c.q[:1]
    q = c.dq[:1].expand(5, -1, -1, -1)
    assert q.stride(0) == 0
    c.check(c.call(q=q))


@FORMATS
@pytest.mark.parametrize("H", [16, 32, 70])
def test_a_query_that_is_not_finite_spoils_no_other(H, fp8):
    c = Case(H, 3, 1, H, 100, [70, 130, 200], 32, fp8)
    c.dq[0, 0, 3, 100], c.dq[1, 0, H - 1, 570], c.dq[2, 0, 0, 0] = float("nan"), float("inf"), -float("inf")
    out = c.call().double().cpu().numpy()
    ref, mag = c.reference()
    spoilt = np.zeros(out.shape[:3], dtype=bool)
    spoilt[0, 0, 3] = spoilt[1, 0, H - 1] = spoilt[2, 0, 0] = True
    assert np.isnan(out[spoilt]).all()
    err = np.abs(out - ref)[~spoilt]
    assert (err <= ((2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(ref))[~spoilt]).all()


@FORMATS
@pytest.mark.parametrize("T,H,prefix", [(130, 1, 0), (65, 3, 0), (33, 16, 50), (200, 2, 0)])
def test_many_tokens(T, H, prefix, fp8):
    # a chunk of a prompt, in one sequence longer and in one shorter than its tokens
    c = Case(T, 3, T, H, prefix, [T + 77, T // 2, T], 16, fp8)
    out = c.call()
    c.check(out)
    if not prefix:
        assert bool((out[1, :T - T // 2] == 0).all())


@FORMATS
@pytest.mark.parametrize("H,prefix", [(16, 0), (32, 0), (70, 0), (16, 300)])
def test_plans_far_longer_than_the_sequences(H, prefix, fp8):
    c = Case(40 + H, 4, 1, H, prefix, [700, 3, 64, 129], 64, fp8)
    wide = torch.full((4, 100000 // 64 + 1), -7, dtype=torch.int32, device="cuda")
    wide[:, :c.d_pages.shape[1]] = c.d_pages
    c.max_len = 100000                              # (what lies behind the lengths names no page)
    c.pages = wide.cpu().numpy()
    c.check(c.call(pages=wide))


@FORMATS
@pytest.mark.parametrize("scale", [0.0, -0.04])
def test_scales_of_zero_and_below(scale, fp8):
    c = Case(50, 2, 1, 20, 90, [130, 7], 32, fp8, scale=scale)
    c.check(c.call())


def test_every_scale_byte():
    # bytes 3 to 254 are exact, what they stand for among bf16's subnormals included; 255 makes its block NaN; rows that the
    # library writes hold 10 to 247
    values = ob.e4m3_values()
    for first in range(0, 256, 32):
        data = np.full((256, 48), 127, dtype=np.uint8)
        data[:, :32], data[:, 32] = np.arange(first, first + 32), np.arange(256)
        out = torch.zeros((256, 32), dtype=torch.bfloat16, device="cuda")
        nmm.nmm_latent_cache_read(torch.from_numpy(data).cuda(), torch.arange(256, device="cuda"), out, kv_lora=32, rope=0)
        got = out.double().cpu().numpy()
        want = values[data[:, :32]] * np.exp2(data[:, 32:33].astype(np.float64) - 127)
        want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
        assert np.array_equal(got[3:255], want[3:255], equal_nan=True), first
        assert np.isnan(got[255]).all()


@pytest.mark.parametrize("M", [1, 2, 4, 8, 9, 32, 40])
@pytest.mark.parametrize("zeros", [False, True])
def test_weights_at_their_zero_points_and_x_with_a_mean(M, zeros):
    # The zero point is taken off a group's sum: the error is a rounding (2^-23 a step, as many as in test_gemv_w4_gpu.py) of
    # sum |x| s (code + zero), also where every code equals it
    K, N, group = 4100, 200, 128
    rng = np.random.default_rng(M)
    x = torch.from_numpy((1 + rng.standard_normal((M, 4104))).astype(np.float32)).to(torch.bfloat16)
    codes = rng.integers(0, 256, (N, 2064), dtype=np.uint8)
    groups = -(-K // group)
    z = rng.integers(0, 16, (N, groups), dtype=np.uint8) if zeros else np.full((N, groups), 8, dtype=np.uint8)
    at = np.repeat(z, group, 1)[:, :4128]
    at = np.pad(at, ((0, 0), (0, 4128 - at.shape[1])))
    codes[::3] = (at[:, 0::2] | (at[:, 1::2] << 4))[::3]                       # rows that stand for nothing but zeros
    scales = torch.from_numpy(rng.uniform(0.002, 0.02, (N, groups)).astype(np.float32)).to(torch.bfloat16)
    y = torch.full((M, N), float("nan"), device="cuda")
    nmm.nmm_gemv_w4(x.cuda(), torch.from_numpy(codes).cuda(), scales.cuda(), y, group=group, K=K,
                    zeros=torch.from_numpy(z).cuda() if zeros else None)
    s, x = scales.double().numpy(), x.double().numpy()[:, :K]
    W = ob.w4_decode(codes, s, group, K, z)
    assert not W[::3].any()
    mag = np.abs(x) @ (np.abs(ob.w4_decode(codes, s, group, K, np.zeros_like(z)))
                       + np.abs(ob.w4_decode(np.zeros_like(codes), s, group, K, z))).T
    err = np.abs(y.double().cpu().numpy() - x @ W.T)
    assert (err <= (8 * 33 + 1 + K / 32 + 4 + 64) * 2.0 ** -23 * mag).all()


def test_the_entry_beside_the_single_tokens():
    # nmm_mla_kv_update rounds fp32 arithmetic's values, this call 64-bit ones: a bf16 step apart at most, and only where fp32's error
    # (2^-18 of a value: a sum of 512 squares and a root; 2^-21 of |k0| + |k1| for RoPE, its angles rounded to fp32) reaches a
    # boundary
    from test_cache_rounding_gpu import entry_of

    kv, rope, hidden, eps, theta = 512, 64, 256, 1e-6, 1e4
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn((1, hidden), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((hidden, kv + rope), generator=g, device="cuda") / 16).to(torch.bfloat16)
    gamma = (1 + 0.1 * torch.randn(kv, generator=g, device="cuda")).to(torch.bfloat16)
    mm = torch.zeros((1, kv + rope), device="cuda")
    one, two = (torch.zeros((64, kv + rope), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for position in (0, 1, 17, 63):
        nmm.nmm_mla_kv_update(h, w, gamma, mm, one, kv_lora=kv, rope=rope, eps=eps, theta=theta, position=position)
        at = torch.tensor([position], device="cuda")
        nmm.nmm_latent_cache_write(mm, at, two, kv_lora=kv, rope=rope, gamma=gamma, eps=eps, positions=at, theta=theta)
        a, b = one[position].double().cpu().numpy(), two[position].double().cpu().numpy()
        exact = ob.cache_entry(mm.double().cpu().numpy(), kv, rope, gamma.double().cpu().numpy(), float(np.float32(eps)), [position],
                               theta)[0]
        k = np.abs(mm[0, kv:].double().cpu().numpy()).reshape(-1, 2).sum(-1).repeat(2)
        off = np.concatenate((2.0 ** -18 * np.abs(exact[:kv]), 2.0 ** -21 * k))
        clear = entry_of(exact - off) == entry_of(exact + off)
        assert clear.sum() > 500 and np.array_equal(a[clear], b[clear])
        # (half a step to each side, and the error)
        assert (np.abs(a - b) <= 2.0 ** -7 * np.abs(exact) + 2 * off).all()
