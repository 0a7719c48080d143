"""nmm_latent_attention_batch against 64-bit attention of every row, over the rows that the cache stands for.

Acceptance per output, derived: each probability is rounded to bf16 (2^-8 relative at most), so the sum moves by at
most 2^-8 sum_j p_j |v_j|; the output's own rounding is 2^-8 |out|; fp32 scores (576 products, |q||k| scale under 64)
move a probability by under 64 * 576 * 2^-24 = 2^-8.8 in the worst case and 2^-12 where the products' signs vary, as here.
"""
import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")


class Case:
    """Inputs of one call: a pool in page order of a permutation, its unused rows NaN."""

    def __init__(self, seed, B, T, H, prefix, lens, page, fp8, kv=512, rope=64, scale=None, max_len=None, sharp=1.0, pad=0):
        rng = np.random.default_rng(seed)
        self.kv, self.rope, self.page, self.prefix, self.lens = kv, rope, page, prefix, np.array(lens, dtype=np.int64)
        self.max_len = int(max(0, max(lens, default=0))) if max_len is None else max_len
        self.scale = (kv + rope) ** -0.5 * sharp if scale is None else scale
        d = kv + rope
        up = lambda n: -(-n // page)
        n_pre, n_own = up(prefix), max(1, up(self.max_len))
        n_pages = n_pre + B * n_own + 2
        order = rng.permutation(n_pages).astype(np.int32)
        self.prefix_pages, self.pages = order[:n_pre], order[n_pre:n_pre + B * n_own].reshape(B, n_own)
        rows = ob.bf16_round(rng.standard_normal((n_pages * page, d)))
        used = np.zeros(n_pages * page, dtype=bool)
        mark = lambda table, n: used.__setitem__(table[np.arange(n) // page] * page + np.arange(n) % page, True)
        mark(self.prefix_pages, prefix)
        for b in range(B):
            mark(self.pages[b], min(max(0, int(self.lens[b])), self.max_len))
        rows[~used] = np.nan
        self.q = ob.bf16_round(rng.standard_normal((B, T, H, d)))
        if fp8:
            data = ob.quantise_rows(rows, kv)
            data[~used, kv:kv + 16] = 255                   # their scales too
            self.values = ob.dequantise_rows(data, kv, rope)
            t = torch.from_numpy(np.pad(data, ((0, 0), (0, pad)), constant_values=0x7F)).cuda()
        else:
            self.values = rows
            t = torch.from_numpy(np.pad(rows, ((0, 0), (0, pad)), constant_values=np.nan).astype(np.float32)).to(torch.bfloat16).cuda()
        self.cache = t
        self.dq = torch.from_numpy(self.q.astype(np.float32)).to(torch.bfloat16).cuda()
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
        self.d_pages, self.d_prefix, self.d_lens = i32(self.pages), i32(self.prefix_pages), i32(self.lens)

    def call(self, out=None, q=None, **kw):
        q = self.dq if q is None else q
        if out is None:
            out = torch.full((*q.shape[:-1], self.kv), float("nan"), dtype=torch.bfloat16, device="cuda")
        args = dict(kv_lora=self.kv, rope=self.rope, page_size=self.page, pages=self.d_pages, lens=self.d_lens,
                    max_len=self.max_len, prefix_pages=self.d_prefix, prefix_len=self.prefix)
        return nmm.nmm_latent_attention_batch(q, self.cache, out, self.scale, **{**args, **kw})

    def reference(self):
        return ob.attention_batch(self.q, self.values, self.scale, self.kv, self.page, self.pages, self.lens, self.max_len,
                                  self.prefix_pages, self.prefix)

    def check(self, out, what=""):
        ref, mag = self.reference()
        o = out.double().cpu().numpy()[..., :self.kv]
        tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(ref)
        bad = ~(np.abs(o - ref) <= tol)
        assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, first {np.argwhere(bad)[0]}: " \
                              f"{o[tuple(np.argwhere(bad)[0])]} for {ref[tuple(np.argwhere(bad)[0])]}"


FORMATS = pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])


@FORMATS
@pytest.mark.parametrize("B,T,H,prefix,lens,page", [
    (1, 1, 1, 0, [1], 64),                     # one position, one row
    (1, 1, 16, 0, [64], 64),                   # one chunk
    (1, 1, 16, 0, [65], 16),                   # one position past it
    (2, 1, 5, 0, [63, 130], 1),                # pages of one row
    (3, 1, 16, 0, [700, 1, 333], 32),          # ragged, some spans empty
    (2, 1, 33, 0, [100, 257], 64),             # rows past a tile of 32
    (2, 1, 128, 0, [300, 77], 128),            # two tiles of 64
    (1, 1, 70, 0, [2000], 256),                # a last tile of 6 rows
    (4, 1, 16, 500, [10, 70, 1, 200], 64),     # a prefix that ends inside a page and a chunk, one tile of 64
    (5, 1, 16, 64, [3, 3, 3, 3, 3], 64),       # 80 rows on the prefix
    (2, 1, 8, 129, [0, 40], 16),               # a sequence with nothing of its own
    (1, 1, 16, 300, [50], 64),                 # the prefix's rows fit one tile
    (2, 2, 16, 100, [2, 90], 32),              # two tokens
    (3, 3, 7, 0, [1, 2, 65], 64),              # tokens that see nothing
    (2, 4, 40, 70, [4, 129], 64),              # four tokens of forty heads
])
def test_shapes(B, T, H, prefix, lens, page, fp8):
    c = Case(B * 100 + H + prefix, B, T, H, prefix, lens, page, fp8)
    c.check(c.call(), f"{B}x{T}x{H}, prefix {prefix}, own {lens}")


@FORMATS
@pytest.mark.parametrize("kv,rope,pad", [(512, 64, 32), (256, 32, 0), (96, 40, 48), (32, 0, 0), (480, 8, 16)])
def test_other_rows(kv, rope, pad, fp8):
    c = Case(kv + rope, 3, 2, 9, 77, [5, 140, 64], 32, fp8, kv=kv, rope=rope, pad=pad)
    c.check(c.call(), f"rows of {kv} + {rope}")


@FORMATS
def test_prefix_alone_and_nothing_at_all(fp8):
    c = Case(5, 3, 1, 20, 333, [0, 0, 0], 64, fp8)
    assert c.max_len == 0
    c.check(c.call(pages=None, lens=None), "prefix alone")
    c.prefix = 0
    out = c.call(pages=None, lens=None, prefix_pages=None)
    assert bool((out == 0).all())


@FORMATS
def test_lengths_outside_the_plan(fp8):
    # above max_len counts as max_len, below zero as zero
    c = Case(6, 4, 1, 16, 0, [5000, -3, 100, 0], 64, fp8, max_len=200)
    out = c.call()
    c.check(out)
    assert bool((out[1] == 0).all()) and bool((out[3] == 0).all())


@FORMATS
@pytest.mark.parametrize("prefix", [0, 200])
def test_pages_outside_the_pool_are_left_out(prefix, fp8):
    c = Case(7, 3, 1, 16, prefix, [150, 64, 100], 16, fp8)
    n = len(c.values) // c.page
    c.pages[0, 2], c.pages[0, 5], c.pages[2, 0] = -1, n, 2 ** 31 - 1
    c.pages[1, :] = -5                                    # a sequence without any page
    if prefix:
        c.prefix_pages[1] = n + 7
    c.d_pages.copy_(torch.from_numpy(c.pages))
    c.d_prefix.copy_(torch.from_numpy(c.prefix_pages))
    out = c.call()
    c.check(out)
    if not prefix:
        assert bool((out[1] == 0).all())


@FORMATS
def test_rising_scores_move_the_reference_every_chunk(fp8):
    c = Case(8, 1, 1, 20, 0, [900], 64, fp8, scale=0.02)
    u = np.sign(np.random.default_rng(2).standard_normal(576))
    rows = c.page * c.pages[0][np.arange(900) // c.page] + np.arange(900) % c.page
    vals = ob.bf16_round(np.random.default_rng(3).standard_normal((900, 576)) * 0.25 + np.linspace(0, 4, 900)[:, None] * u)
    c.q = ob.bf16_round(np.abs(c.q) * u)
    c.dq.copy_(torch.from_numpy(c.q.astype(np.float32)))
    if fp8:
        data = ob.quantise_rows(vals, 512)
        c.cache[torch.from_numpy(rows).cuda()] = torch.from_numpy(data).cuda()
        vals = ob.dequantise_rows(data, 512, 64)
    else:
        c.cache[torch.from_numpy(rows).cuda()] = torch.from_numpy(vals.astype(np.float32)).to(torch.bfloat16).cuda()
    c.values[rows] = vals
    c.check(c.call())


@FORMATS
def test_sharp_softmax_and_the_same_bits_again(fp8):
    c = Case(9, 4, 1, 32, 1000, [100, 300, 7, 900], 64, fp8, sharp=12.0)
    a = c.call()
    # scores up to 12 times larger: their fp32 rounding counts for 12 * 2^-12
    ref, mag = c.reference()
    err = np.abs(a.double().cpu().numpy() - ref)
    assert np.all(err <= (2.0 ** -8 + 12 * 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(ref))
    for _ in range(3):
        assert torch.equal(c.call(), a)


def test_strided_queries_and_outputs():
    c = Case(10, 3, 2, 12, 90, [60, 2, 130], 32, True)
    wide = torch.full((2, 12, 3, 640), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = wide.permute(2, 0, 1, 3)                          # [batch, tokens, heads, 640], heads 3 rows apart
    q[..., :576] = c.dq
    big = torch.full((3, 12, 2, 528), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big.permute(0, 2, 1, 3)
    c.call(out=out, q=q)
    c.check(out)
    assert bool((big[..., 512:] == 7.0).all())


def test_three_dimensional_queries():
    c = Case(11, 5, 1, 16, 0, [20, 30, 40, 50, 60], 64, False)
    c.check(c.call(q=c.dq[:, 0])[:, None])


@FORMATS
def test_rows_past_32_bit_offsets(fp8):
    # a pool of 5 GB whose sequences lie at its ends and across 2^31 and 2^32 bytes
    ld, page, kv = 2048, 64, 512
    rows = (5 << 30) // ld
    data = torch.empty((rows, ld), dtype=torch.uint8, device="cuda")
    cache = data if fp8 else data.view(torch.bfloat16)
    at = [0, (1 << 31) // ld // page - 1, (1 << 32) // ld // page - 1, rows // page - 2]
    pages = torch.tensor([[a, a + 1] for a in at], dtype=torch.int32, device="cuda")
    lens = [128, 100, 65, 127]
    vals = ob.bf16_round(np.random.default_rng(1).standard_normal((4, 128, 576)))
    slots = torch.cat([torch.arange(a * page, (a + 2) * page) for a in at]).cuda()
    src = torch.from_numpy(vals.reshape(-1, 576).astype(np.float32)).cuda()
    nmm.nmm_latent_cache_write(src, slots, cache, kv_lora=kv, rope=64)
    if fp8:
        vals = ob.dequantise_rows(ob.quantise_rows(vals.reshape(-1, 576), kv), kv, 64)
    q = ob.bf16_round(np.random.default_rng(2).standard_normal((4, 1, 16, 576)))
    out = torch.zeros((4, 1, 16, kv), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_latent_attention_batch(torch.from_numpy(q.astype(np.float32)).to(torch.bfloat16).cuda(), cache, out, 0.07, kv_lora=kv,
                                   rope=64, page_size=page, pages=pages, max_len=128,
                                   lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    ref, mag = ob.attention_batch(q, vals.reshape(-1, 576), 0.07, kv, page, np.arange(8).reshape(4, 2), lens, 128)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert np.all(err <= (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(ref))


@FORMATS
def test_random_batches(fp8):
    rng = np.random.default_rng(77 + fp8)
    for k in range(10):
        B, T = int(rng.integers(1, 9)), int(rng.choice([1, 1, 2, 3]))
        H = int(rng.integers(1, 130 // T))
        prefix = int(rng.choice([0, rng.integers(1, 1500)]))
        lens = rng.integers(0, 600, B).tolist()
        page = int(rng.choice([1, 8, 16, 64, 128]))
        print(f"case {k}: {B}x{T}x{H} prefix {prefix} own {lens} page {page}", flush=True)
        c = Case(1000 + k, B, T, H, prefix, lens, page, fp8)
        c.check(c.call(), f"case {k}")


def test_captured_call_follows_lengths_and_pages():
    c = Case(12, 4, 1, 16, 150, [300, 300, 300, 300], 64, True)
    out = torch.zeros((4, 1, 16, 512), dtype=torch.bfloat16, device="cuda")
    ws = nmm.Workspace()
    c.call(out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(out=out, workspace=ws)
    for lens in ([300, 1, 64, 0], [2, 299, 128, 65], [300, 300, 300, 300]):
        c.lens = np.array(lens)
        c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.pages = np.ascontiguousarray(np.roll(c.pages, 1, axis=0))
        c.d_pages.copy_(torch.from_numpy(c.pages))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        c.call(out=out)
        torch.cuda.synchronize()
        assert torch.equal(replayed, out), lens
        c.check(out)


def test_two_streams_with_their_own_workspaces():
    a = Case(13, 2, 1, 16, 400, [100, 500], 64, True)
    b = Case(14, 3, 1, 128, 0, [300, 200, 100], 64, False)
    want = a.call(), b.call()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        outs = [torch.zeros_like(w) for w in want]
        torch.cuda.synchronize()
        a.call(out=outs[0], stream=s1)
        b.call(out=outs[1], stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_python_refusals():
    c = Case(20, 2, 1, 4, 40, [30, 40], 16, True, kv=64, rope=32)
    c.call()
    half = c.dq.half()
    for bad in (dict(q=half), dict(out=torch.zeros((2, 1, 4, 64), device="cuda")), dict(q=c.dq[0, 0])):
        with pytest.raises(TypeError):
            c.call(**bad)
    ok = torch.zeros((2, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(out=ok[:1]), dict(out=ok[..., :63]), dict(q=c.dq[..., :95], out=ok), dict(pages=None), dict(lens=None), dict(lens=c.d_lens[:1]),
                dict(pages=c.d_pages[:, :1]), dict(pages=c.d_pages.long()), dict(lens=c.d_lens.long()), dict(prefix_pages=None),
                dict(prefix_pages=c.d_prefix[:1]), dict(page_size=24), dict(page_size=0), dict(max_len=-1), dict(prefix_len=-1),
                dict(kv_lora=48, out=ok), dict(rope=12), dict(lens=c.d_lens.cpu()), dict(kv_lora=512, out=ok)):
        with pytest.raises((ValueError, nmm.NmmError)):                 # the binding's checks, the library's
            c.call(**bad)


@FORMATS
def test_a_sequence_whose_row_is_nan_spoils_no_other(fp8):
    c = Case(21, 4, 1, 16, 90, [70, 3, 129, 1], 16, fp8)
    at = int(c.pages[1, 0]) * 16 + 2
    if fp8:
        c.cache[at, 5] = 0x7F
    else:
        c.cache[at, 5] = float("nan")
    out = c.call()
    assert bool(torch.isnan(out[1]).any())
    ref, mag = c.reference()
    o = out.double().cpu().numpy()
    keep = [0, 2, 3]
    assert (np.abs(o[keep] - ref[keep]) <= (2.0 ** -8 + 2.0 ** -12) * mag[keep] + 2.0 ** -8 * np.abs(ref[keep])).all()
