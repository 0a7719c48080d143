"""nmm_latent_attention_batch over pools whose byte offsets pass 2^31 and 2^32, in every size of tile: pages at the pool's ends and
on both sides of 2^31 and 2^32 bytes in one table, pages outside the pool among them, spans of many chunks.  Tolerances as in
test_attention_batch_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

KV, ROPE, PAGE, LD = 512, 64, 16, 2048
ROWS = (5 << 30) // LD
N_PAGES = ROWS // PAGE


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("B,T,H,prefix,lens", [
    (3, 1, 16, 0, [700, 333, 129]),                                      # tiles of 16 rows
    (4, 1, 32, 0, [1000, 517, 64, 1]),                                   # of 32
    (40, 1, 32, 0, [500 - 11 * b for b in range(40)]),                   # of 32, spans of several chunks
    (2, 2, 16, 0, [900, 65]),                                            # of 32, two tokens
    (3, 1, 64, 0, [900, 500, 63]),                                       # of 64
    (4, 1, 40, 0, [0, 30, 64, 0]),                                       # of 64, one span: sequences of no position
    (16, 1, 128, 2000, [100, 1, 33, 64] * 4),                            # of 64, the prefix in spans of many chunks
    (128, 1, 64, 0, [640 - 3 * b for b in range(128)]),                  # of 64, own positions in spans of many chunks
])
def test_pool_of_five_gigabytes(B, T, H, prefix, lens, fp8):
    rng = np.random.default_rng(B + H + prefix)
    up = lambda n: -(-n // PAGE)
    longest = max(lens)
    n_pre, n_own = up(prefix), up(longest)
    need = n_pre + B * n_own
    # the pages of the pool that are used: a quarter each from its start, its end and around 2^31 and 2^32 bytes
    part = -(-need // 4)
    page31, page32 = (1 << 31) // LD // PAGE, (1 << 32) // LD // PAGE
    ids = np.concatenate((np.arange(part), page31 - part // 2 + np.arange(part), page32 - part // 2 + np.arange(part),
                          N_PAGES - part + np.arange(part)))
    assert len(np.unique(ids)) == len(ids) and ids.min() == 0 and ids.max() == N_PAGES - 1
    order = rng.permutation(len(ids))[:need].astype(np.int64)            # compact page numbers
    prefix_pages, pages = order[:n_pre].copy(), order[n_pre:].reshape(B, n_own).copy()
    vals = ob.bf16_round(rng.standard_normal((len(ids) * PAGE, KV + ROPE)))
    pool = torch.empty((ROWS, LD), dtype=torch.uint8, device="cuda")
    cache = pool if fp8 else pool.view(torch.bfloat16)
    slots = (ids[:, None] * PAGE + np.arange(PAGE)).reshape(-1)
    nmm.nmm_latent_cache_write(torch.from_numpy(vals.astype(np.float32)).cuda(), torch.from_numpy(slots).cuda(), cache, kv_lora=KV,
                               rope=ROPE)
    if fp8:
        vals = ob.dequantise_rows(ob.quantise_rows(vals, KV), KV, ROPE)
    # pages outside the pool: before, just behind and far behind it
    for table in (pages, prefix_pages[None]):
        for k, bad in enumerate((-1, -(1 << 31), -2, -3)):
            if table.shape[1] > 4 * k + 3:
                table[k % len(table), 4 * k + 3] = bad
    outside = {-1: -1, -2: N_PAGES, -3: (1 << 31) - 1, -(1 << 31): -(1 << 31)}
    device = lambda t: torch.tensor([outside[v] if v < 0 else int(ids[v]) for v in t.reshape(-1).tolist()], dtype=torch.int32,
                                    device="cuda").view(t.shape)
    q = ob.bf16_round(rng.standard_normal((B, T, H, KV + ROPE)))
    out = torch.full((B, T, H, KV), float("nan"), dtype=torch.bfloat16, device="cuda")
    scale = (KV + ROPE) ** -0.5
    print(f"{B}x{T}x{H} prefix {prefix}, {'8-bit' if fp8 else 'bf16'} rows", flush=True)
    nmm.nmm_latent_attention_batch(torch.from_numpy(q.astype(np.float32)).to(torch.bfloat16).cuda(), cache, out, scale, kv_lora=KV,
                                   rope=ROPE, page_size=PAGE, pages=device(pages), max_len=longest,
                                   lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), prefix_pages=device(prefix_pages),
                                   prefix_len=prefix)
    ref, mag = ob.attention_batch(q, vals, scale, KV, PAGE, pages, lens, longest, prefix_pages, prefix)
    err = np.abs(out.double().cpu().numpy() - ref)
    bad = ~(err <= (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(ref))
    assert not bad.any(), f"{bad.sum()} of {bad.size} outside, first {np.argwhere(bad)[0]}"
