"""The feed-forward half of a decode step as a layer runs it: the router's logits, the choice of experts, the expert that every token
takes (two products with an epilogue, the second onto the residual stream) and the chosen experts' sum onto that.

Each stage is compared with 64-bit arithmetic on the values that the stage before it left, so that each tolerance is one
stage's: the products' and the experts' as oracle/ffn.py derives them, the choice equal.
"""
import numpy as np
import pytest
import torch

from oracle import ffn

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

HIDDEN, INNER, SHARED, E, K = 264, 96, 160, 32, 4
HALF = 2.0 ** -8
SILU = nmm.NMM_ACT_SILU


class Layer:
    def __init__(self, seed, T, first=0, local=E):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape, sigma=1.0: (torch.randn(shape, generator=g, device="cuda") * sigma).to(torch.bfloat16)
        self.T, self.first, self.g = T, first, g
        self.w_gate = normal(E, HIDDEN, sigma=HIDDEN ** -0.5)
        self.bias = torch.randn(E, generator=g, device="cuda") * 0.05
        self.w1 = normal(local, 2 * INNER, HIDDEN, sigma=HIDDEN ** -0.5)
        self.w2 = normal(local, HIDDEN, INNER, sigma=INNER ** -0.5)
        self.s1, self.s2 = normal(2 * SHARED, HIDDEN, sigma=HIDDEN ** -0.5), normal(HIDDEN, SHARED, sigma=SHARED ** -0.5)
        self.x = torch.zeros((T, HIDDEN), dtype=torch.bfloat16, device="cuda")          # the normalised stream
        self.stream = torch.zeros((T, HIDDEN), dtype=torch.bfloat16, device="cuda")
        self.mask = torch.ones(T, dtype=torch.uint8, device="cuda")
        self.logits = torch.zeros((T, E), device="cuda")
        self.h = torch.zeros((T, SHARED), dtype=torch.bfloat16, device="cuda")
        self.mid, self.out = torch.zeros_like(self.stream), torch.zeros_like(self.stream)
        self.route = (torch.zeros((T, K), dtype=torch.int32, device="cuda"), torch.zeros((T, K), device="cuda"),
                      torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(T * K, dtype=torch.int32, device="cuda"))
        self.ws = nmm.Workspace()

    def next_tokens(self, padded=0.0):
        self.x.copy_(torch.randn((self.T, HIDDEN), generator=self.g, device="cuda"))
        self.stream.copy_(torch.randn((self.T, HIDDEN), generator=self.g, device="cuda"))
        self.mask.copy_(torch.rand(self.T, generator=self.g, device="cuda") >= padded)

    def run(self):
        ws = self.ws
        nmm.nmm_gemv_nt(self.x, self.w_gate, self.logits, workspace=ws)
        nmm.nmm_moe_route(self.logits, *self.route, score=nmm.NMM_SCORE_SIGMOID, bias=self.bias, groups=4, top_groups=2, group_top=2,
                          renormalize=True, scale=2.5, mask=self.mask, workspace=ws)
        nmm.nmm_gemv_nt_act(self.x, self.s1, self.h, act=SILU, gated=True, workspace=ws)
        nmm.nmm_gemv_nt_act(self.h, self.s2, self.mid, residual=self.stream, workspace=ws)
        nmm.nmm_moe_experts(self.x, self.w1, self.w2, *self.route, self.out, first=self.first, residual=self.mid, workspace=ws)

    def check(self):
        up = lambda t: t.double().cpu().numpy()
        x = up(self.x)
        ref, mag = x @ up(self.w_gate).T, np.abs(x) @ np.abs(up(self.w_gate)).T
        assert (np.abs(up(self.logits) - ref) <= (HIDDEN + 33 * (HIDDEN / 32 + 1)) * 2.0 ** -24 * mag).all()
        chosen, w, offsets, pairs = ffn.route(up(self.logits), K, False, up(self.bias), 4, 2, 2, True, 2.5, self.mask.cpu().numpy())
        got = [t.cpu().numpy() for t in self.route]
        assert np.array_equal(got[0], chosen) and np.array_equal(got[2], offsets) and np.array_equal(got[3][:len(pairs)], pairs)
        assert (np.abs(got[1] - w) <= 2.0 ** -24 * w + 2.0 ** -50).all()

        def near(y, ref, err):
            assert (np.abs(up(y) - ref) <= err + HALF * (np.abs(ref) + err)).all()

        near(self.h, *ffn.nt_act(x, up(self.s1), SILU, True))
        near(self.mid, *ffn.nt_act(up(self.h), up(self.s2), 0, False, residual=up(self.stream)))
        near(self.out, *ffn.experts(x, up(self.w1), up(self.w2), got[0], got[1], self.first, SILU, HALF, up(self.mid)))


@pytest.mark.parametrize("T,first,local", [(1, 0, E), (7, 0, E), (20, 8, 16), (70, 0, E), (300, 24, 8)])
def test_layers_one_after_the_other(T, first, local):
    layer = Layer(T, T, first, local)
    for padded in (0.0, 0.4, 1.0):
        layer.next_tokens(padded)
        layer.run()
        torch.cuda.synchronize()
        layer.check()


@pytest.mark.parametrize("T", [1, 24, 100, 400])
def test_a_captured_layer_serves_every_token(T):
    layer = Layer(T + 1, T)
    layer.next_tokens()
    layer.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run()
    for i in range(5):
        layer.next_tokens(0.2 * i)
        graph.replay()
        torch.cuda.synchronize()
        layer.check()
        got = layer.out.clone(), layer.route[0].clone()
        layer.out.zero_()
        layer.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], layer.out) and torch.equal(got[1], layer.route[0]), i


def test_two_layers_on_two_streams():
    """Calls that may overlap, each stream with its own workspaces: the results of the same calls one after the other."""
    a, b = Layer(1, 90), Layer(2, 33)
    a.ws = b.ws = None
    for layer in (a, b):
        layer.next_tokens()
        layer.run()
    torch.cuda.synchronize()
    ref = a.out.clone(), b.out.clone()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for layer in (a, b):
        layer.out.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, s in ((a, streams[0]), (b, streams[1])):
            with torch.cuda.stream(s):
                layer.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out, ref[0]) and torch.equal(b.out, ref[1])
