"""The batched operators as a decode batch runs them: the cache entry's and the queries' products from 4-bit weights, the
cache rows, attention over them behind a shared prefix, and the output projection, for tokens one after the other.

Each stage is compared with 64-bit arithmetic on the values that the stage before it left, so that each tolerance is
one stage's: 4-bit products as in test_gemv_w4_gpu.py, cache rows equal (their inputs are the products'), attention as in
test_attention_batch_gpu.py.
"""
import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

HIDDEN, KV, ROPE, HEADS, PAGE, EPS, THETA = 320, 128, 32, 6, 16, 1e-6, 1e4
D = KV + ROPE


class W4:
    def __init__(self, rng, N, K, group, mx):
        self.group, self.K = group, K
        self.codes = rng.integers(0, 256, (N, (K + 31) // 32 * 16), dtype=np.uint8)
        if mx:
            scales = rng.integers(121, 124, (N, -(-K // group)), dtype=np.uint8)
            self.scales = torch.from_numpy(scales).cuda()
        else:
            self.scales = torch.from_numpy(rng.uniform(0.01, 0.03, (N, -(-K // group)))).to(torch.bfloat16).cuda()
            scales = self.scales.double().cpu().numpy()
        self.W = ob.w4_decode(self.codes, scales, group, K, None, mx)
        self.most = np.abs(self.W) if mx else np.abs(self.W) + 16 * np.repeat(scales, group, 1)[:, :K]
        self.codes = torch.from_numpy(self.codes).cuda()

    def __call__(self, x, y, ws=None):
        return nmm.nmm_gemv_w4(x, self.codes, self.scales, y, group=self.group, K=self.K, workspace=ws)

    def check(self, x, y):
        x = x.double().cpu().numpy()
        bad = ~(np.abs(y.double().cpu().numpy() - x @ self.W.T) <= (8 * 33 + 1 + self.K / 32 + 68) * 2.0 ** -23 * (np.abs(x) @ self.most.T))
        assert not bad.any()


class Step:
    """One token of every sequence."""

    def __init__(self, seed, B, prefix, longest, fp8):
        rng = np.random.default_rng(seed)
        self.B, self.prefix, self.fp8, self.longest = B, prefix, fp8, longest
        self.w_entry, self.w_q = W4(rng, D, HIDDEN, 64, False), W4(rng, HEADS * D, HIDDEN, 32, True)
        self.w_o = W4(rng, HIDDEN, HEADS * KV, 128, False)
        n_pre, n_own = -(-prefix // PAGE), -(-longest // PAGE)
        order = rng.permutation(n_pre + B * n_own + 1).astype(np.int32)
        self.pages = order[n_pre:n_pre + B * n_own].reshape(B, n_own)
        self.prefix_pages = order[:n_pre]
        rows = len(order) * PAGE
        width = nmm.nmm_latent_cache_row_bytes(KV, ROPE) if fp8 else D
        self.cache = torch.zeros((rows, width), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda")
        at = (self.prefix_pages[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:prefix]
        src = torch.from_numpy(rng.standard_normal((prefix, D)).astype(np.float32)).cuda()
        if prefix:
            nmm.nmm_latent_cache_write(src, torch.from_numpy(at.astype(np.int64)).cuda(), self.cache, kv_lora=KV, rope=ROPE)
        self.gamma = (1 + 0.1 * torch.randn(KV, device="cuda")).to(torch.bfloat16)
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
        self.d_pages, self.d_prefix = i32(self.pages), i32(self.prefix_pages)
        self.x = torch.zeros((B, HIDDEN), dtype=torch.bfloat16, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.slots = torch.full((B,), -1, dtype=torch.int64, device="cuda")
        self.positions = torch.zeros(B, dtype=torch.int64, device="cuda")
        self.entry = torch.zeros((B, D), device="cuda")
        self.q32 = torch.zeros((B, HEADS * D), device="cuda")
        self.q = torch.zeros((B, HEADS, D), dtype=torch.bfloat16, device="cuda")
        self.o = torch.zeros((B, HEADS, KV), dtype=torch.bfloat16, device="cuda")
        self.y = torch.zeros((B, HIDDEN), device="cuda")
        self.ws = nmm.Workspace()

    def next_token(self, seed, idle=()):
        """Inputs of the next token; sequences named in idle have none (padding: slot -1, nothing appended)."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.x.copy_(torch.randn((self.B, HIDDEN), generator=g, device="cuda"))
        lens = self.lens.cpu().numpy()
        slots = np.full(self.B, -1, dtype=np.int64)
        for b in range(self.B):
            if b not in idle:
                slots[b] = self.pages[b, lens[b] // PAGE] * PAGE + lens[b] % PAGE
                lens[b] += 1
        self.slots.copy_(torch.from_numpy(slots))
        self.lens.copy_(torch.from_numpy(lens))
        self.positions.copy_(torch.from_numpy(self.prefix + lens.astype(np.int64) - 1).clamp(min=0))

    def run(self):
        self.w_entry(self.x, self.entry, self.ws)
        nmm.nmm_latent_cache_write(self.entry, self.slots, self.cache, kv_lora=KV, rope=ROPE, gamma=self.gamma, eps=EPS,
                                   positions=self.positions, theta=THETA)
        self.w_q(self.x, self.q32, self.ws)
        self.q.copy_(self.q32.view(self.B, HEADS, D))
        nmm.nmm_latent_attention_batch(self.q, self.cache, self.o, D ** -0.5, kv_lora=KV, rope=ROPE, page_size=PAGE,
                                       pages=self.d_pages, lens=self.lens, max_len=self.longest,
                                       prefix_pages=self.d_prefix, prefix_len=self.prefix, workspace=self.ws)
        self.w_o(self.o.view(self.B, HEADS * KV), self.y, self.ws)

    def rows(self):
        if self.fp8:
            return ob.dequantise_rows(self.cache.cpu().numpy(), KV, ROPE)
        return self.cache.double().cpu().numpy()

    def check(self, before):
        self.w_entry.check(self.x, self.entry)
        rows, slots = self.rows(), self.slots.cpu().numpy()
        live = slots >= 0
        entry = ob.cache_entry(self.entry.double().cpu().numpy(), KV, ROPE, self.gamma.double().cpu().numpy(), EPS,
                               self.positions.cpu().numpy(), THETA)
        # the entry's rounding to bf16 and, for latents, to e4m3 may fall the other way: 2^-8 and 2^-4 of the value, 2^-10
        # times 2^-4 of the block's largest for e4m3's subnormals
        top = np.abs(entry[:, :KV]).reshape(self.B, -1, 32).max(-1).repeat(32, 1)
        tol = np.abs(entry) * 2.0 ** -7 + 1e-5
        if self.fp8:
            tol[:, :KV] += np.abs(entry[:, :KV]) * 2.0 ** -3 + top * 2.0 ** -14
        assert (np.abs(rows[slots[live]] - entry[live]) <= tol[live]).all()
        others = np.setdiff1d(np.arange(rows.shape[0]), slots)
        assert torch.equal(self.cache[torch.from_numpy(others)], before[torch.from_numpy(others)])
        self.w_q.check(self.x, self.q32)
        lens = self.lens.cpu().numpy().astype(np.int64)
        ref, mag = ob.attention_batch(self.q.double().cpu().numpy()[:, None], rows, D ** -0.5, KV, PAGE, self.pages, lens, self.longest,
                                      self.prefix_pages, self.prefix)
        o = self.o.double().cpu().numpy()[:, None]
        assert (np.abs(o - ref) <= (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(ref)).all()
        self.w_o.check(self.o.view(self.B, HEADS * KV), self.y)


@pytest.mark.parametrize("B,prefix,fp8", [(1, 0, True), (5, 100, True), (9, 300, False), (20, 33, True)])
def test_tokens_one_after_the_other(B, prefix, fp8):
    s = Step(B, B, prefix, 40, fp8)
    for t in range(4):
        s.next_token(10 * B + t, idle=() if t != 2 else (0,))
        before = s.cache.clone()
        s.run()
        torch.cuda.synchronize()
        s.check(before)


def test_a_captured_step_serves_every_token():
    s = Step(3, 6, 70, 64, True)
    s.next_token(0)
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for t in range(1, 20):
        s.next_token(t, idle=(t % 7,))
        before = s.cache.clone()
        graph.replay()
        torch.cuda.synchronize()
        s.check(before)
        got = s.y.clone(), s.o.clone(), s.cache.clone()
        s.cache.copy_(before)
        s.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], s.y) and torch.equal(got[1], s.o) and torch.equal(got[2], s.cache), t
