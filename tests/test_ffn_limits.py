"""Sizes that the header of the feed-forward operators allows are not refused, those past its limits are; without a GPU."""
import ctypes
import os

import pytest

nmm = pytest.importorskip("paper_2609_16009_amd")
if not os.path.exists(nmm.LIB_PATH):
    pytest.skip("libnmm.so not built", allow_module_level=True)

L = nmm.lib()
A = 1 << 34          # fake addresses, never dereferenced here


def experts(**kw):
    """The status of a call on an expert of hidden x inner weights, without a workspace."""
    d = dict(tokens=16, top_k=1, experts=4, first=0, local=4, hidden=8, inner=8, dt=nmm.NMM_BF16, act=nmm.NMM_ACT_SILU, x=A, W1=2 * A,
             W2=3 * A, chosen=4 * A, weights=4 * A, offsets=4 * A, pairs=4 * A, residual=None, y=5 * A)
    d.update(kw)
    up8 = lambda n: (n + 7) // 8 * 8
    for k, v in dict(ldx=up8(d["hidden"]), ldw1=up8(d["hidden"]), ldw2=up8(d["inner"]), ldy=d["hidden"], ldr=d["hidden"]).items():
        d.setdefault(k, v)
    d.setdefault("stride1", 2 * d["inner"] * d["ldw1"])
    d.setdefault("stride2", d["hidden"] * d["ldw2"])
    s = nmm.nmm_moe_ffn()
    for k, v in d.items():
        setattr(s, k, v)
    return L.nmm_moe_experts(ctypes.byref(s), None, 0, None)


@pytest.mark.parametrize("tokens,top_k,hidden", [(1 << 24, 1, 8), ((1 << 26) - 1, 1, 8), ((1 << 24) + 1, 3, 16), (1 << 24, 2, 56), (1 << 20, 32, 1000),
                                                 ((1 << 25) - 1, 1, 24)])
def test_as_many_tokens_as_the_header_says(tokens, top_k, hidden):
    """Only the workspace is missing."""
    assert experts(tokens=tokens, top_k=top_k, hidden=hidden) == nmm.NMM_ERR_WORKSPACE


@pytest.mark.parametrize("kw", [dict(tokens=1 << 26), dict(tokens=1 << 25, top_k=2), dict(tokens=1 << 25, hidden=32),
                                dict(hidden=1 << 29, local=0), dict(inner=1 << 29, local=0), dict(ldy=1 << 31)])
def test_past_the_header(kw):
    assert experts(**kw) == nmm.NMM_ERR_SHAPE


@pytest.mark.parametrize("T,inner", [(300, 1 << 23), (16, (1 << 26) - 1), (100000, (1 << 26) - 1)])
def test_long_rows_of_h_are_allowed(T, inner):
    assert experts(tokens=T, inner=inner, experts=1, local=1) == nmm.NMM_ERR_WORKSPACE
