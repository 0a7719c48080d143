"""What nmm_latent_cache_write rounds RMSNorm's and RoPE's results to: the 64-bit formula's value, rounded to the nearest float and
that to the nearest bf16 number (ties to even, both), as torch casts a double to bfloat16.  Every entry is compared, but for those
whose rounding what the kernel's fp64 may be off by would change:

RMSNorm 2^-40 of the value (16 levels of sums, the inverse root's Newton step from an fp32 one, 1.5 * (2^-22)^2, two products);
RoPE 2^-33 of |k0| + |k1| at positions below 2^17 (the angle: 2 j 2^-53 of pos * theta^(-2 j / rope), j theta^(-2 j / rope) at most
1.3 here, and the product's and its reduction's own rounding, 2^-36, twice: the kernel's and the oracle's)."""
import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

FORMATS = pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])


def entry_of(exact):
    return ob.bf16_round(np.asarray(exact, dtype=np.float64).astype(np.float32))


def errors(src, exact, kv):
    """What the kernel's fp64 may be off by."""
    k = np.abs(np.asarray(src, dtype=np.float64)[:, kv:]).reshape(len(src), -1, 2).sum(-1).repeat(2, 1)
    return np.concatenate((2.0 ** -40 * np.abs(exact[:, :kv]), 2.0 ** -33 * k), 1)


def written(src, kv, rope, fp8, gamma=None, eps=0.0, pos=None, theta=1e4):
    """The rows' bytes."""
    n = len(src)
    width = nmm.nmm_latent_cache_row_bytes(kv, rope, nmm.NMM_CACHE_E4M3 if fp8 else nmm.NMM_CACHE_BF16)
    cache = torch.zeros((n, width), dtype=torch.uint8, device="cuda")
    g = None if gamma is None else torch.from_numpy(gamma.astype(np.float32)).to(torch.bfloat16).cuda()
    p = None if pos is None else torch.from_numpy(np.asarray(pos, dtype=np.int64)).cuda()
    nmm.nmm_latent_cache_write(torch.from_numpy(src).cuda(), torch.arange(n, device="cuda"),
                               cache if fp8 else cache.view(torch.bfloat16), kv_lora=kv, rope=rope, gamma=g, eps=float(eps),
                               positions=p, theta=theta)
    return cache.cpu().numpy()


def rows_of(entry, kv, fp8):
    return ob.quantise_rows(entry, kv) if fp8 else ob.bf16_encode(entry).view(np.uint8).reshape(len(entry), -1)


def in_floats(src, kv, rope, gamma, eps, pos, theta):
    """The entry by a row's arithmetic in fp32."""
    f = np.float32
    c, k = src[:, :kv], src[:, kv:]
    c = c * (f(1) / np.sqrt((c * c).mean(1, dtype=f, keepdims=True) + f(eps))) * gamma.astype(f)
    a = (pos[:, None] * float(theta) ** (-2.0 * np.arange(rope // 2) / rope)) % (2 * np.pi)
    cs, sn = np.cos(a).astype(f), np.sin(a).astype(f)
    k = np.stack((k[:, 0::2] * cs - k[:, 1::2] * sn, k[:, 0::2] * sn + k[:, 1::2] * cs), -1).reshape(k.shape)
    return ob.bf16_round(np.concatenate((c, k), 1))


@FORMATS
def test_every_entry(fp8):
    kv, rope, theta, tokens = 512, 64, 1e4, 8192
    eps = np.float32(1e-6)
    rng = np.random.default_rng(31)
    src = rng.standard_normal((tokens, kv + rope)).astype(np.float32)
    gamma = ob.bf16_round(1 + 0.1 * rng.standard_normal(kv))
    pos = rng.integers(0, 2 ** 17, tokens)
    exact = ob.cache_entry(src, kv, rope, gamma, float(eps), pos, theta)
    off, entry = errors(src, exact, kv), entry_of(exact)
    sure = entry_of(exact - off) == entry_of(exact + off)
    assert (~sure).sum() <= 8                                   # about 2^-24 of the RoPE values
    # fp32 arithmetic would move dozens of entries, and rows with them
    assert ((in_floats(src, kv, rope, gamma, eps, pos, theta) != entry) & sure).sum() >= 20
    got, want = written(src, kv, rope, fp8, gamma, eps, pos, theta), rows_of(entry, kv, fp8)
    # bytes that only sure entries decide: two a value, or a block of 32 codes and its scale
    if fp8:
        block = sure[:, :kv].reshape(tokens, -1, 32).all(-1)
        clear = np.concatenate((block.repeat(32, 1), block, np.ones((tokens, 16 - kv // 32), bool), sure[:, kv:].repeat(2, 1)), 1)
    else:
        clear = sure.repeat(2, 1)
    wrong = (got != want) & clear
    assert not wrong.any(), f"{wrong.sum()} bytes, first {np.argwhere(wrong)[0]}"


TIES = [1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 1.5 + 2.0 ** -8, 1.5 + 3 * 2.0 ** -8]     # two whose even neighbour is below, two above


@FORMATS
def test_rope_beside_a_tie(fp8):
    # pair 3 of 4 turns by pos * 10^-12: k0 cos - k1 sin is a tie of bf16 plus or minus that.  Within half a float step of the tie,
    # 2^-24, it goes to even like the tie, further off to its own side
    kv, rope = 32, 8
    src, pos = [], []
    for tie in TIES:
        for k1 in (-1.0, 1.0):
            for sign in (-1.0, 1.0):
                for p in (1, 100, 10000, 100000, 1000000):
                    row = np.zeros(kv + rope)
                    row[-2:] = sign * tie, k1
                    src.append(row)
                    pos.append(p)
    src, pos = np.array(src, dtype=np.float32), np.array(pos)
    exact = ob.cache_entry(src, kv, rope, None, 0.0, pos, 1e16)
    entry = entry_of(exact)
    even = entry_of(src)[:, -2] == entry[:, -2]
    assert even[pos <= 10000].all() and even[pos >= 100000].mean() == 0.5
    assert np.array_equal(written(src, kv, rope, fp8, pos=pos, theta=1e16)[:, -4:], rows_of(entry, kv, fp8)[:, -4:])


@FORMATS
@pytest.mark.parametrize("bits", [31, 21])
def test_norm_beside_a_tie(bits, fp8):
    # mean(c^2) + eps = 1 + 2^-bits in exactly representable terms: the latent c_0, a tie, is normalised to c_0 (1 - 2^-(bits + 1)),
    # within half a float step of the tie or below it
    kv = 32
    for tie in TIES[:2]:
        for sign in (-1.0, 1.0):
            src = np.zeros((1, kv), dtype=np.float32)
            src[0, 0], src[0, 1] = sign * tie, 2.0 ** ((5 - bits) / 2)
            eps = 1 - tie * tie / kv
            assert float(np.float32(eps)) == eps
            assert (src.astype(np.float64) ** 2).sum() / kv + eps == 1 + 2.0 ** -bits
            exact = ob.cache_entry(src, kv, 0, np.ones(kv), eps)
            entry = entry_of(exact)
            assert abs(entry[0, 0]) == (tie - 2.0 ** -8 if bits == 21 or tie == TIES[0] else tie + 2.0 ** -8)
            assert np.array_equal(written(src, kv, 0, fp8, np.ones(kv), eps), rows_of(entry, kv, fp8)), (tie, sign)


@pytest.mark.parametrize("B,prefix,fp8", [(5, 100, True), (9, 300, False)])
def test_a_steps_rows(B, prefix, fp8):
    # the rows that a decode batch's step writes, from the products it took: byte for byte
    from test_batch_step_gpu import EPS, KV, ROPE, THETA, Step

    s = Step(B, B, prefix, 40, fp8)
    gamma = s.gamma.double().cpu().numpy()
    for t in range(3):
        s.next_token(50 * B + t)
        s.run()
        torch.cuda.synchronize()
        src, pos, slots = s.entry.double().cpu().numpy(), s.positions.cpu().numpy(), s.slots.cpu().numpy()
        exact = ob.cache_entry(src, KV, ROPE, gamma, float(np.float32(EPS)), pos, THETA)
        off = errors(src, exact, KV)
        sure = entry_of(exact - off) == entry_of(exact + off)
        assert (~sure).sum() <= 1
        got = s.cache[torch.from_numpy(slots).cuda()].view(torch.uint8).cpu().numpy()
        rows = sure.all(1)
        assert np.array_equal(got[rows], rows_of(entry_of(exact), KV, fp8)[rows])
