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
