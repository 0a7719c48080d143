"""The largest sizes that nmm_moe_experts takes.

Weights are zero but for a few columns of h, the first and last among them, so that the reference is small and every sum an exact
integer: results must be equal, after one rounding to bf16.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

GIB = 1 << 30
TICKETS = 65536


def integers(g, *shape, dtype=torch.bfloat16):
    return torch.randint(-1, 2, shape, generator=g, device="cuda").to(dtype)


def stale(nbytes):
    """A workspace whose counters are zero and whose other bytes are NaN in either type."""
    ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:TICKETS] = 0
    return ws


def one_expert(T):
    """A choice of the only expert by every token, weight 1."""
    i32 = dict(dtype=torch.int32, device="cuda")
    return (torch.zeros((T, 1), **i32), torch.ones((T, 1), device="cuda"), torch.tensor([0, T], **i32), torch.arange(T, **i32))


@pytest.mark.parametrize("T,inner", [(300, 1 << 23), (300, (1 << 22) + 5), (100, (1 << 23) + 9), (16, (1 << 26) - 1), (12, (1 << 26) - 9)])
def test_rows_of_h_that_add_up_to_gigabytes(T, inner):
    """256, 128, 64 and 16 rows of h past 2^31 and 2^32 bytes: y is every row's sum, not its residual alone."""
    hidden, up8 = 8, (inner + 7) // 8 * 8
    g = torch.Generator(device="cuda").manual_seed(T)
    at = torch.tensor([0, 7, 64, 12345, inner // 2, inner // 2 + 3, inner - 9, inner - 1], device="cuda")
    w1 = torch.zeros((1, 2 * inner, hidden), dtype=torch.bfloat16, device="cuda")
    w2 = torch.zeros((1, hidden, up8), dtype=torch.bfloat16, device="cuda")
    gate, up, down = integers(g, 8, hidden), integers(g, 8, hidden), integers(g, hidden, 8)
    w1[0, at], w1[0, inner + at] = gate, up
    w2[0, :, inner:] = float("nan")                    # behind the last column: nobody's
    w2[0][:, at] = down
    x, residual = integers(g, T, hidden), integers(g, T, hidden)
    y = torch.full((T, hidden), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = stale(TICKETS + T * ((inner + 63) // 64 * 128 + 32) + 512)
    nmm.nmm_moe_experts(x, w1, w2, *one_expert(T), y, act=nmm.NMM_ACT_RELU, inner=inner, residual=residual, workspace=ws)
    x, gate, up, down = (t.double().cpu() for t in (x, gate, up, down))
    h = (x @ gate.T).clamp(min=0) * (x @ up.T)
    want = (residual.double().cpu() + h @ down.T).to(torch.bfloat16)
    assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("T,top_k,hidden", [((1 << 24) + 77, 1, 8), ((1 << 23) + 5, 2, 17)])
def test_tokens_past_a_launch_of_the_sums(T, top_k, hidden):
    """More blocks than a launch of the sums has: each token's are there, and nothing beside them."""
    inner, up8 = 8, (hidden + 7) // 8 * 8
    g = torch.Generator(device="cuda").manual_seed(top_k)
    w1, w2 = integers(g, 2, 2 * inner, up8), integers(g, 2, hidden, inner)
    x = integers(g, T, up8)
    i32 = dict(dtype=torch.int32, device="cuda")
    chosen = torch.randint(0, 2, (T, 1), generator=g, **i32) if top_k == 1 else torch.randint(0, 2, (T, 1), generator=g, **i32) ^ torch.arange(2, **i32)
    flat = chosen.reshape(-1)
    offsets = torch.zeros(3, **i32)
    offsets[1:] = torch.cumsum(torch.bincount(flat, minlength=2), 0)
    pairs = torch.sort(flat, stable=True)[1].to(torch.int32)
    weights = torch.tensor([0.5, 2.0], device="cuda")[torch.randint(0, 2, (T, top_k), generator=g, device="cuda")]
    residual = integers(g, T, hidden)
    whole = torch.full((T + 2, hidden), 7.0, dtype=torch.bfloat16, device="cuda")
    nmm.nmm_moe_experts(x, w1, w2, chosen, weights, offsets, pairs, whole[1:-1], act=nmm.NMM_ACT_NONE, hidden=hidden, residual=residual)
    assert (whole[0] == 7).all() and (whole[-1] == 7).all()
    # integers of 2^20 at most: fp32 holds every sum
    want = residual.float()
    for e in range(2):
        z = x[:, :hidden].float() @ w1[e, :, :hidden].float().T
        h = (z[:, :inner] * z[:, inner:]).to(torch.bfloat16).float()
        want += (h @ w2[e].float().T) * torch.where(chosen == e, weights, 0.0).sum(1, keepdim=True)
    assert torch.equal(whole[1:-1], want.to(torch.bfloat16))
