"""nmm_latent_cache_write / nmm_latent_cache_read against the 64-bit formulas: rows byte for byte where the
entry has no arithmetic before its rounding, within a rounding of bf16 and e4m3 where it has."""
import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def pool(rows, kv, rope, fp8, pad=0, fill=0xA5):
    n = nmm.nmm_latent_cache_row_bytes(kv, rope, nmm.NMM_CACHE_E4M3 if fp8 else nmm.NMM_CACHE_BF16) + pad
    t = torch.full((rows, n), fill, dtype=torch.uint8, device="cuda")
    return t if fp8 else t.view(torch.bfloat16)


def special_rows(kv, rope, seed=3):
    """bf16 rows with what a block's scale can go wrong at: zeros, one value, the border 448 * 2^e from both sides, ties
    between codes, the smallest and largest exponents, infinities and NaN."""
    rng = np.random.default_rng(seed)
    r = ob.bf16_round(rng.standard_normal((12, kv + rope)) * np.exp2(rng.integers(-30, 30, (12, 1))))
    r[0, :kv] = 0
    r[1, :32] = 0
    r[1, 5] = 448.0
    r[2, :32] = 450.0                                      # just above 448: the next exponent
    r[3, :16], r[3, 16:32] = 1.0, 1.0625                   # 1.0625 is halfway between two codes
    r[4, :32] = 2.0 ** -126
    r[5, :32] = 2.0 ** -133                                # a subnormal bf16
    r[6, :32] = 3.3895313892515355e38
    r[7, 3], r[7, 9], r[7, 12] = np.inf, -np.inf, np.nan
    r[8, :32] = np.inf                                     # a block with no finite value
    r[9, :kv] = ob.bf16_round(np.exp2(rng.integers(-24, 1, kv) * 1.0) * rng.choice([-1, 1], kv))   # codes below normal
    return r


@pytest.mark.parametrize("src32", [True, False])
@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("kv,rope", [(512, 64), (256, 32), (32, 8), (480, 0), (96, 40)])
def test_rows_byte_for_byte(kv, rope, fp8, src32):
    r = special_rows(kv, rope)
    if not fp8:
        r[np.isnan(r)] = 1.0                               # a bf16 NaN's payload is not compared
    n = len(r)
    src = torch.from_numpy(r.astype(np.float32))
    src = src.cuda() if src32 else src.to(torch.bfloat16).cuda()
    cache = pool(40, kv, rope, fp8, pad=32)
    before = cache.clone()
    slots = torch.from_numpy(np.random.default_rng(1).permutation(40)[:n].astype(np.int64)).cuda()
    nmm.nmm_latent_cache_write(src, slots, cache, kv_lora=kv, rope=rope)
    got = cache.view(torch.uint8).cpu().numpy()
    width = nmm.nmm_latent_cache_row_bytes(kv, rope, 2 if fp8 else 1)
    ref = ob.quantise_rows(r, kv) if fp8 else ob.bf16_encode(r).view(np.uint8).reshape(n, -1)
    at = slots.cpu().numpy()
    nan = got[at, :kv] & 127 == 127 if fp8 else None
    if fp8:                                                # a NaN keeps no sign
        ref[:, :kv][nan & (ref[:, :kv] == 127)] = got[at, :kv][nan & (ref[:, :kv] == 127)]
    assert np.array_equal(got[at, :width], ref)
    # the padding of the written rows and every other row, as they were
    keep = before.view(torch.uint8).cpu().numpy()
    assert np.array_equal(got[:, width:], keep[:, width:])
    others = np.setdiff1d(np.arange(40), at)
    assert np.array_equal(got[others], keep[others])
    # read back: what the rows stand for, exactly
    out = torch.full((n, kv + rope + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    nmm.nmm_latent_cache_read(cache, slots, out, kv_lora=kv, rope=rope)
    want = ob.dequantise_rows(ref, kv, rope) if fp8 else r
    o = out.double().cpu().numpy()
    assert np.array_equal(o[:, :kv + rope], want, equal_nan=True)
    assert np.all(o[:, kv + rope:] == 3.0)


@pytest.mark.parametrize("tokens", [1, 3, 64, 1027])
@pytest.mark.parametrize("fp8", [True, False])
def test_entries_with_norm_and_rope(tokens, fp8):
    kv, rope, eps, theta = 512, 64, 1e-6, 10000.0
    rng = np.random.default_rng(tokens)
    down = rng.standard_normal((tokens, 64 + kv + rope)).astype(np.float32)     # the wider product's columns
    gamma = ob.bf16_round(1 + 0.1 * rng.standard_normal(kv))
    pos = rng.integers(0, 2 ** 31, tokens)
    pos[0] = 0
    cache = pool(2048, kv, rope, fp8)
    slots = rng.permutation(2048)[:tokens]
    dev = torch.from_numpy(down).cuda()
    nmm.nmm_latent_cache_write(dev[:, 64:], torch.from_numpy(slots).cuda(), cache, kv_lora=kv, rope=rope,
                               gamma=bf16(gamma).cuda(), eps=eps, positions=torch.from_numpy(pos).cuda(), theta=theta)
    out = torch.zeros((tokens, kv + rope), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_latent_cache_read(cache, torch.from_numpy(slots).cuda(), out, kv_lora=kv, rope=rope)
    exact = ob.cache_entry(down[:, 64:], kv, rope, gamma, eps, pos, theta)
    o = out.double().cpu().numpy()
    # one rounding to bf16 (2^-8 relative at most) of fp32 arithmetic on values of order one; the fp32 part: a sum of
    # 512 squares and a root (2^-20), and angles reduced in fp64 but rounded to fp32 (2^-23 absolute)
    assert np.all(np.abs(o[:, kv:] - exact[:, kv:]) <= 2.0 ** -8 * np.abs(exact[:, kv:]) + 2.0 ** -20 * 8)
    entry = ob.bf16_round(exact)
    tol = 2.0 ** -8 * np.abs(exact[:, :kv]) * (1 + 2.0 ** -8)
    if fp8:
        # and one to e4m3: half a step, 2^-4 relative, or 2^-10 of the block's scale below the normal codes
        amax = np.abs(entry[:, :kv]).reshape(tokens, -1, 32).max(-1).repeat(32, 1)
        tol = tol + np.maximum(2.0 ** -4 * np.abs(exact[:, :kv]) * (1 + 2.0 ** -7), 2.0 ** -10 * amax / 224)
        # and nearly all rows byte for byte: a code differs only where fp32 and 64 bits round to different bf16 values
        ref = ob.quantise_rows(entry, kv)
        same = (cache.cpu().numpy()[slots] == ref).mean()
        assert same > 0.999, same
    assert np.all(np.abs(o[:, :kv] - exact[:, :kv]) <= tol + 1e-30)


def test_norm_alone_and_rope_alone():
    kv, rope = 128, 16
    rng = np.random.default_rng(8)
    x = rng.standard_normal((5, kv + rope)).astype(np.float32)
    gamma, pos = ob.bf16_round(1 + 0.1 * rng.standard_normal(kv)), np.arange(5) * 1000
    slots = torch.arange(5, device="cuda")
    for kw, ref in ((dict(gamma=bf16(gamma).cuda(), eps=0.5), ob.cache_entry(x, kv, rope, gamma, 0.5)),
                    (dict(positions=torch.from_numpy(pos).cuda(), theta=500.0),
                     ob.cache_entry(x, kv, rope, None, 0, pos, 500.0))):
        cache = pool(5, kv, rope, False)
        nmm.nmm_latent_cache_write(torch.from_numpy(x).cuda(), slots, cache, kv_lora=kv, rope=rope, **kw)
        got = cache.double().cpu().numpy()
        assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -20)


@pytest.mark.parametrize("fp8", [True, False])
def test_slots_outside_are_skipped_and_reads_repeat(fp8):
    kv, rope = 64, 8
    cache = pool(6, kv, rope, fp8)
    keep = cache.view(torch.uint8).clone()
    src = torch.randn((7, kv + rope), device="cuda")
    out_of = torch.tensor([-1, 6, 1 << 40, -(1 << 62), 6, 100, -7], device="cuda")
    nmm.nmm_latent_cache_write(src, out_of, cache, kv_lora=kv, rope=rope)
    assert torch.equal(cache.view(torch.uint8), keep)
    out = torch.full((7, kv + rope), 2.0, dtype=torch.bfloat16, device="cuda")
    nmm.nmm_latent_cache_read(cache, out_of, out, kv_lora=kv, rope=rope)
    assert bool((out == 2.0).all())
    slots = torch.tensor([4, -1, 0, 2, 9, 5, -1], device="cuda")
    nmm.nmm_latent_cache_write(src, slots, cache, kv_lora=kv, rope=rope)
    now = cache.view(torch.uint8)
    assert torch.equal(now[[1, 3]], keep[[1, 3]]) and not torch.equal(now[[0, 2, 4, 5]], keep[[0, 2, 4, 5]])
    twice = torch.tensor([4, 4, -1, 0, 4, 0, 2], device="cuda")
    nmm.nmm_latent_cache_read(cache, twice, out, kv_lora=kv, rope=rope)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[4]) and torch.equal(out[3], out[5])
    assert bool((out[2] == 2.0).all())


@pytest.mark.parametrize("fp8", [True, False])
def test_rows_past_32_bit_offsets(fp8):
    # a pool of 5 GB: rows whose byte offsets pass 2^31 and 2^32
    kv, rope, ld = 512, 64, 2048
    rows = (5 << 30) // ld
    data = torch.empty((rows, ld), dtype=torch.uint8, device="cuda")
    cache = data if fp8 else data.view(torch.bfloat16)
    slots = torch.tensor([0, (1 << 31) // ld - 1, (1 << 31) // ld, (1 << 32) // ld, rows - 1], device="cuda")
    src = torch.randn((5, kv + rope), device="cuda").to(torch.bfloat16)
    out = torch.zeros((5, kv + rope), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_latent_cache_write(src, slots, cache, kv_lora=kv, rope=rope)
    nmm.nmm_latent_cache_read(cache, slots, out, kv_lora=kv, rope=rope)
    ref = src.double().cpu().numpy()
    if fp8:
        ref = ob.dequantise_rows(ob.quantise_rows(ref, kv), kv, rope)
    assert np.array_equal(out.double().cpu().numpy(), ref)


def test_other_stream_and_graph_replays():
    kv, rope = 512, 64
    cache = pool(64, kv, rope, True)
    src, slots = torch.randn((16, kv + rope), device="cuda"), torch.arange(16, device="cuda") * 3
    out = torch.zeros((16, kv + rope), dtype=torch.bfloat16, device="cuda")

    def step():
        nmm.nmm_latent_cache_write(src, slots, cache, kv_lora=kv, rope=rope)
        nmm.nmm_latent_cache_read(cache, slots, out, kv_lora=kv, rope=rope)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        src.normal_()
        slots.copy_((torch.arange(16, device="cuda") * 3 + i) % 64)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        step()
        assert torch.equal(replayed, out), i


@pytest.mark.parametrize("fp8", [True, False])
def test_entries_are_rounded_once(fp8):
    # RMSNorm and RoPE are in fp64 (their angles below 2^17 to 2^-35) up to a float that is rounded to bf16: it ends on the wrong side
    # of one of bf16's boundaries where the value is within half a float step of it, 2^-17 of the values; four times that are
    # allowed (in fp32, with errors around 2^-23, twice as many would be wrong)
    kv, rope, eps, theta, tokens = 512, 64, 1e-6, 10000.0, 2048
    rng = np.random.default_rng(31)
    src = rng.standard_normal((tokens, kv + rope)).astype(np.float32)
    gamma = ob.bf16_round(1 + 0.1 * rng.standard_normal(kv))
    pos = rng.integers(0, 2 ** 17, tokens)
    cache = pool(tokens, kv, rope, fp8)
    slots = torch.arange(tokens, device="cuda")
    nmm.nmm_latent_cache_write(torch.from_numpy(src).cuda(), slots, cache, kv_lora=kv, rope=rope, gamma=bf16(gamma).cuda(), eps=eps,
                               positions=torch.from_numpy(pos).cuda(), theta=theta)
    out = torch.zeros((tokens, kv + rope), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_latent_cache_read(cache, slots, out, kv_lora=kv, rope=rope)
    entry = ob.bf16_round(ob.cache_entry(src, kv, rope, gamma, eps, pos, theta))
    if fp8:
        entry = ob.dequantise_rows(ob.quantise_rows(entry, kv), kv, rope)
    wrong = (out.double().cpu().numpy() != entry).mean()
    assert wrong <= 2.0 ** -15, wrong
