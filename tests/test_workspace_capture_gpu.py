"""Workspaces that a captured call grows: its counters are zeroed by the graph itself, and only when that graph is replayed, so
no other graph and no eager call may count on them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

M, K, N, GROUP = 4, 16384, 96, 32                          # K split over workgroups: counters and partial sums


class Product:
    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
        self.w = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8, device="cuda")
        self.s = torch.rand((N, K // GROUP), generator=g, device="cuda").to(torch.bfloat16)
        self.y = torch.zeros((M, N), device="cuda")
        self.want = self.run(torch.empty_like(self.y), nmm.Workspace()).clone()
        torch.cuda.synchronize()

    def run(self, y, ws, stream=None):
        return nmm.nmm_gemv_w4(self.x, self.w, self.s, y, group=GROUP, workspace=ws, stream=stream)

    def check(self, run, what):
        self.y.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        same = torch.equal(self.y, self.want)
        assert same, what


@pytest.fixture
def fresh(monkeypatch):
    monkeypatch.setattr(nmm, "_default_ws", {})


def capture(product, ws, stream, times=1):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(times):
            product.run(product.y, ws)
    return graph


def dirty(given):
    """What memory may hold that nothing has initialised yet, in every buffer of the workspaces."""
    for ws in [given] if given else list(nmm._default_ws.values()):
        for buf in [ws.buf, *ws._retired]:
            buf.fill_(0x55)
    torch.cuda.synchronize()


@pytest.mark.parametrize("given", [False, True], ids=["default", "given"])
def test_two_graphs_replayed_in_either_order(given, fresh):
    assert nmm.lib().nmm_gemv_w4_workspace_size(M, K, N, GROUP) > 0
    ws, stream = nmm.Workspace() if given else None, torch.cuda.Stream()
    a, b = Product(1), Product(2)
    ga, gb = capture(a, ws, stream), capture(b, ws, stream, times=2)
    dirty(ws)
    for _ in range(3):
        b.check(gb.replay, "the second graph")
        a.check(ga.replay, "the first graph")


@pytest.mark.parametrize("given", [False, True], ids=["default", "given"])
def test_an_eager_call_before_the_first_replay(given, fresh):
    ws, stream = nmm.Workspace() if given else None, torch.cuda.Stream()
    a, b = Product(3), Product(4)
    graph = capture(a, ws, stream)
    dirty(ws)
    for _ in range(3):
        with torch.cuda.stream(stream):
            b.check(lambda: b.run(b.y, ws), "the eager call")
        a.check(graph.replay, "the graph")
    # and a graph captured after it
    later = capture(b, ws, stream)
    for _ in range(3):
        b.check(later.replay, "the later graph")
        a.check(graph.replay, "the graph")


def test_captures_are_told_apart():
    stream, ids = torch.cuda.Stream(), []
    x = torch.zeros(8, device="cuda")
    for _ in range(3):
        assert nmm._capture_id(stream.cuda_stream) == 0
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            x.add_(1)
            ids.append(nmm._capture_id(stream.cuda_stream))
            x.add_(1)
            assert nmm._capture_id(stream.cuda_stream) == ids[-1]
            assert nmm._capture_id(0) == 0
    assert 0 not in ids and len(set(ids)) == 3


def test_a_capture_behind_a_warm_up_shares_the_buffer(fresh):
    # what an eager call has zeroed serves graphs too, and a capture that needs more gets its own
    ws, stream = nmm.Workspace(), torch.cuda.Stream()
    a, b = Product(5), Product(6)
    with torch.cuda.stream(stream):
        a.check(lambda: a.run(a.y, ws), "eager")
    held = ws.held
    graphs = [(p, capture(p, ws, stream)) for p in (a, b)]
    assert ws.held == held and not ws._retired
    for _ in range(3):
        for p, graph in reversed(graphs):
            p.check(graph.replay, "a graph")
        with torch.cuda.stream(stream):
            b.check(lambda: b.run(b.y, ws), "eager")
    graph = torch.cuda.CUDAGraph()
    big, y = torch.randn((32, K), device="cuda").to(torch.bfloat16), torch.zeros((32, 7168), device="cuda")
    codes = torch.randint(0, 256, (7168, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.rand((7168, K // GROUP), device="cuda").to(torch.bfloat16)
    want = nmm.nmm_gemv_w4(big, codes, scales, torch.zeros_like(y), group=GROUP, workspace=nmm.Workspace())
    assert nmm.lib().nmm_gemv_w4_workspace_size(32, K, 7168, GROUP) > held[1]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        nmm.nmm_gemv_w4(big, codes, scales, y, group=GROUP, workspace=ws)
        a.run(a.y, ws)
    for _ in range(3):
        with torch.cuda.stream(stream):
            b.check(lambda: b.run(b.y, ws), "eager")
        y.fill_(float("nan"))
        a.check(graph.replay, "the capture that grew the workspace")
        same = torch.equal(y, want)
        assert same
        for p, g in graphs:
            p.check(g.replay, "an older graph")
