"""nmm_gemv_nt_act against its formula in 64 bits (oracle/ffn.py derives the bound of what fp32 sums may be off).

Small integers make every sum exact, so those results must be equal, after one rounding to the output's type.
"""
import numpy as np
import pytest
import torch

from oracle import ffn

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}           # half a step of the subnormals


def make(seed, M, K, N, gated, dt, integer, bias, residual, pad=0, sigma=1.0):
    """Device tensors and their values; past K everything is NaN, which may not reach a result."""
    rng = np.random.default_rng(seed)
    rows = 2 * N if gated else N

    def tensor(shape, width, scale):
        v = rng.integers(-3, 4, shape) if integer else rng.standard_normal(shape) * scale
        full = np.full((*shape[:-1], width), np.nan)
        full[..., :shape[-1]] = v
        t = torch.from_numpy(full.astype(np.float32)).to(dt)
        return t.cuda(), t[..., :shape[-1]].double().numpy()

    up8 = (K + 7) // 8 * 8 + 8 * pad
    x, xv = tensor((M, K), up8, sigma)
    Wt, wv = tensor((rows, K), up8 + 16 * pad, 1.0 if integer else K ** -0.5)
    b, bv = tensor((rows,), rows, 0.5) if bias else (None, None)
    r, rv = tensor((M, N), N + 5 * pad, 1.0) if residual else (None, None)
    return dict(x=x, Wt=Wt, bias=b, residual=None if r is None else r[:, :N]), (xv, wv, bv, rv)


def rounded(v, dt):
    return torch.from_numpy(np.ascontiguousarray(v)).to(dt).double().numpy()


def check(seed, M, K, N, act=0, gated=False, dt=torch.bfloat16, integer=False, bias=False, residual=False, pad=0, sigma=1.0, **kw):
    args, (x, w, b, r) = make(seed, M, K, N, gated, dt, integer, bias, residual, pad, sigma)
    y = torch.full((M, N + 3), 7.0, dtype=dt, device="cuda")
    y32 = torch.full((M, N + 2), 7.0, device="cuda")
    nmm.nmm_gemv_nt_act(args.pop("x"), args.pop("Wt"), y[:, :N], K=K, act=act, gated=gated, y_f32=y32[:, :N], **args, **kw)
    assert (y[:, N:] == 7).all() and (y32[:, N:] == 7).all(), "columns past N"
    got, got32 = y[:, :N].double().cpu().numpy(), y32[:, :N].double().cpu().numpy()
    ref, err = ffn.nt_act(x, w, act, gated, b, r)
    what = (M, K, N, ffn.ACTS[act], gated, dt, bias, residual)
    if integer:
        assert np.array_equal(got32, ref), what
        assert np.array_equal(got, rounded(ref.astype(np.float32), dt)), what
        return
    bad = ~(np.abs(got32 - ref) <= err)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first {np.argwhere(bad)[0]}: {got32[bad][0]} for {ref[bad][0]}"
    # the 16-bit output is the fp32 one, rounded once
    assert np.array_equal(got, rounded(got32.astype(np.float32), dt)), what


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
def test_integers_exact_at_every_row_count(dt, act, gated):
    for M in (1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 64, 65, 100, 128, 129, 257):
        check(M, M, 137, 70, act, gated, dt, True, bias=M % 2 == 0, residual=M % 3 == 0)


@pytest.mark.parametrize("M", [1, 7, 16, 33, 130])
@pytest.mark.parametrize("K,N", [(1, 1), (7, 17), (8, 16), (31, 15), (64, 32), (127, 33), (128, 5), (129, 100), (255, 48), (512, 130),
                                 (1000, 257), (4099, 31)])
def test_integers_exact_at_odd_sizes(M, K, N):
    check(K + N, M, K, N, 1, False, torch.bfloat16, True, bias=True, residual=True)
    check(K + N, M, K, N, 0, True, torch.float16, True, bias=True, residual=True, pad=1)


@pytest.mark.parametrize("M,K,N", [(33, 1024, 70), (64, 1031, 257), (65, 1500, 129), (128, 4099, 100), (129, 2048, 33), (200, 3000, 1000),
                                   (300, 512, 2100), (1000, 600, 40), (5, 2048, 100), (20, 4096, 300), (2, 6144, 4100), (31, 2048, 8200)])
def test_integers_exact_where_k_is_cut_or_walks_start_apart(M, K, N):
    """K in one, two, four and eight slices, ending within a chunk of 8 and on one; rows of the weight 4 KB apart and not."""
    check(M + K, M, K, N, 1, False, torch.bfloat16, True, bias=True, residual=M % 2 == 0)
    check(M + N, M, K, N, 0, True, torch.float16, True, residual=M % 2 == 1)


def test_one_workspace_for_every_size():
    ws = nmm.Workspace()
    for M, K, N in ((256, 2048, 300), (40, 1024, 100), (1, 512, 64), (128, 4096, 200), (300, 700, 30), (256, 2048, 300)):
        check(M + K, M, K, N, 1, M % 3 == 0, torch.bfloat16, True, residual=True, workspace=ws)


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_every_activation(act, gated, dt):
    for M, K, N in ((1, 520, 200), (6, 333, 77), (24, 1536, 64), (70, 264, 130)):
        check(act + M, M, K, N, act, gated, dt, bias=True, residual=M > 1)
    check(act, 9, 128, 300, act, gated, dt, sigma=12.0)      # far into both tails


@pytest.mark.parametrize("M,K,N,gated", [(1, 7168, 512, True), (32, 16384, 130, False), (256, 2048, 300, True), (300, 1001, 517, False),
                                         (64, 4096, 1024, True)])
def test_large_products(M, K, N, gated):
    check(M, M, K, N, 2, gated, residual=True, pad=1)


def test_activations_at_the_ends():
    """Infinities, NaN and zeros of either sign through the epilogue: x is the identity's row, so z is the weight."""
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 88.0, -88.0, 1e30, -1e30, float("inf"), float("-inf"), float("nan"), 3e38])
    Wt = torch.zeros((12, 8), dtype=torch.bfloat16)
    Wt[:, 0] = v
    x = torch.zeros((1, 8), dtype=torch.bfloat16)
    x[0, 0] = 1
    for act in range(5):
        y = torch.zeros((1, 12), device="cuda")
        nmm.nmm_gemv_nt_act(x.cuda(), Wt.cuda(), None, act=act, y_f32=y)
        got, ref = y[0].double().cpu().numpy(), ffn.activation(Wt[:, 0].double().numpy(), act)
        finite = np.isfinite(ref)
        if act >= 3:          # z^3 and e^-z leave fp32's range before 64 bits': what is left is 0, z, or NaN at -inf
            finite &= np.abs(ref) < 1e37
        assert np.allclose(got[finite], ref[finite], rtol=1e-5, atol=1e-37), ffn.ACTS[act]
        assert np.isnan(got[10]) and got[8] == np.inf, ffn.ACTS[act]
        if act == 1:
            assert got[9] == 0


@pytest.mark.parametrize("M", [1, 8, 20, 100])
def test_a_value_that_is_not_finite_stays_in_its_row(M):
    args, (x, w, _, _) = make(M, M, 300, 90, True, torch.bfloat16, False, False, False)
    clean = torch.zeros((M, 90), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], clean, K=300, act=2, gated=True)
    hurt = M // 2
    args["x"][hurt, 17] = float("nan")
    args["Wt"][5, 3] = float("inf")
    y = torch.zeros_like(clean)
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], y, K=300, act=2, gated=True)
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[hurt], keep[:, 5] = False, False
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[hurt]).all()


@pytest.mark.parametrize("M,K", [(70, 128), (200, 2048)])
def test_residual_in_place_in_wide_tiles(M, K):
    args, _ = make(M, M, K, 130, False, torch.bfloat16, False, True, True)
    y = torch.zeros((M, 130), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], y, act=4, bias=args["bias"], residual=args["residual"])
    both = args["residual"].clone()
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], both, act=4, bias=args["bias"], residual=both)
    assert torch.equal(both, y)


def test_residual_in_place_and_column_ranges():
    args, (x, w, _, r) = make(3, 21, 256, 64, False, torch.bfloat16, False, False, True)
    y = torch.zeros((21, 64), dtype=torch.bfloat16, device="cuda")
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], y, act=3, residual=args["residual"])
    both = args["residual"].clone()
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], both, act=3, residual=both)
    assert torch.equal(both, y)
    # x, the residual and y as column ranges of one buffer
    buf = torch.zeros((21, 256 + 64 + 64), dtype=torch.bfloat16, device="cuda")
    buf[:, :256], buf[:, 256:320] = args["x"], args["residual"]
    nmm.nmm_gemv_nt_act(buf[:, :256], args["Wt"], buf[:, 320:], act=3, residual=buf[:, 256:320])
    assert torch.equal(buf[:, 320:], y) and torch.equal(buf[:, :256], args["x"])
    with pytest.raises(nmm.NmmError, match="NMM_ERR_ARG"):
        nmm.nmm_gemv_nt_act(buf[:, :256], args["Wt"], buf[:, 310:374], act=3, residual=buf[:, 256:320])


def test_no_products_leave_the_epilogue():
    b = torch.randn(40, device="cuda").to(torch.float16)
    r = torch.randn((3, 40), device="cuda").to(torch.float16)
    x, Wt = torch.zeros((3, 8), dtype=torch.float16, device="cuda"), torch.zeros((40, 8), dtype=torch.float16, device="cuda")
    y = torch.zeros((3, 40), dtype=torch.float16, device="cuda")
    nmm.nmm_gemv_nt_act(x, Wt, y, K=0, act=1, bias=b, residual=r)
    ref = torch.relu(b.float()) + r.float()
    assert torch.equal(y, ref.half())
    empty = torch.zeros((0, 40), dtype=torch.float16, device="cuda")
    assert nmm.nmm_gemv_nt_act(x[:0], Wt, empty) is empty


def test_agrees_with_nmm_gemv_nt():
    x = torch.randn((7, 1536), device="cuda").to(torch.bfloat16)
    Wt = (torch.randn((300, 1536), device="cuda") / 40).to(torch.bfloat16)
    a, b = torch.zeros((7, 300), device="cuda"), torch.zeros((7, 300), device="cuda")
    nmm.nmm_gemv_nt(x, Wt, a)
    nmm.nmm_gemv_nt_act(x, Wt, None, y_f32=b)
    mag = x.double().abs() @ Wt.double().abs().T
    assert ((a.double() - b.double()).abs() <= (1536 + 33 * 49 + 16) * 2.0 ** -24 * mag + 2.0 ** -23 * a.abs()).all()


@pytest.mark.parametrize("M", [1, 12, 40, 200])
def test_streams_captures_and_repeats(M):
    args, _ = make(M, M, 1000, 260, True, torch.bfloat16, False, True, True)
    call = lambda y, **kw: nmm.nmm_gemv_nt_act(args["x"], args["Wt"], y, K=1000, act=2, gated=True, bias=args["bias"],
                                               residual=args["residual"], **kw)
    y = [torch.zeros((M, 260), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    call(y[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call(y[1], stream=s)
    with torch.cuda.stream(s):
        call(y[2])
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y[3])
    for i in range(4):
        args["x"].mul_(-1)
        y[3].zero_()
        graph.replay()
        call(y[0])
        torch.cuda.synchronize()
        assert torch.equal(y[3], y[0]), i


def test_binding_refuses():
    x, Wt = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((32, 64), dtype=torch.bfloat16, device="cuda")
    y, f = torch.zeros((2, 32), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 32), device="cuda")
    act = nmm.nmm_gemv_nt_act
    for bad in (lambda: act(x.float(), Wt, y), lambda: act(x, Wt.half(), y), lambda: act(x, Wt, f), lambda: act(x, Wt, y, y_f32=y)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: act(x, Wt, None), lambda: act(x, Wt, y[:1]), lambda: act(x, Wt, y[:, :16]), lambda: act(x, Wt, y, gated=True),
                lambda: act(x, Wt, y, K=65), lambda: act(x, Wt, y, bias=x[0]), lambda: act(x, Wt, y, bias=f[0]),
                lambda: act(x, Wt, y, residual=f), lambda: act(x, Wt, y, residual=y[:1]), lambda: act(x, Wt, y, y_f32=f[:1]),
                lambda: act(x.cpu(), Wt, y), lambda: act(x.t(), Wt, y), lambda: act(x[0], Wt, y)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(nmm.NmmError, match="NMM_ERR_ARG"):
        act(x, Wt, y, act=9)


# Tiles of 64 and of 128 rows: K past 4096, or weights of many rows.
@pytest.mark.parametrize("K", [4097, 4104, 4160, 4223, 4224, 5000, 8192])
@pytest.mark.parametrize("M,N", [(33, 1), (48, 70), (64, 128), (65, 129), (130, 200), (257, 63)])
def test_integers_exact_in_tiles_of_64(M, N, K):
    check(M + K, M, K, N, 1, False, torch.bfloat16, True, bias=True, residual=M % 2 == 0, pad=K % 2)
    check(M + N, M, K, N, 0, True, torch.float16, True, residual=M % 2 == 1)


@pytest.mark.parametrize("M,N,K", [(129, 2900, 2100), (200, 2177, 2056), (400, 5000, 1), (400, 5000, 65), (257, 8000, 130), (400, 4990, 192),
                                   (1000, 1100, 300), (300, 4100, 2304)])
def test_integers_exact_in_tiles_of_128(M, N, K):
    check(M + K, M, K, N, 1, False, torch.bfloat16, True, bias=True, residual=True)
    check(M + K, M, K, N // 2, 0, True, torch.float16, True, residual=True, pad=1)


@pytest.mark.parametrize("M,N", [(70, 300), (129, 2900)])
@pytest.mark.parametrize("gated", [False, True])
def test_every_activation_in_tiles(M, N, gated):
    for act in range(5):
        check(act, M, 4110 if M == 70 else 2060, N, act, gated, torch.float16 if act % 2 else torch.bfloat16, bias=True, residual=True)


@pytest.mark.parametrize("M,K,N", [(70, 4200, 260), (300, 2300, 2100), (400, 64, 2501)])
def test_tiles_in_place_on_streams_and_captured(M, K, N):
    args, _ = make(M, M, K, N, True, torch.bfloat16, False, True, True)
    call = lambda y, r, **kw: nmm.nmm_gemv_nt_act(args["x"], args["Wt"], y, K=K, act=2, gated=True, bias=args["bias"], residual=r, **kw)
    ref = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    call(ref, args["residual"])
    y = args["residual"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call(y, y, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y, args["residual"])
    for i in range(4):
        args["x"].mul_(-1)
        y.zero_()
        graph.replay()
        call(ref, args["residual"])
        torch.cuda.synchronize()
        assert torch.equal(y, ref), i


@pytest.mark.parametrize("M,N", [(100, 40), (400, 5000)])
def test_a_value_that_is_not_finite_stays_in_its_row_of_a_tile(M, N):
    K = 4300 if M == 100 else 140
    args, _ = make(M, M, K, N, True, torch.bfloat16, False, False, False)
    clean, y = (torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], clean, K=K, act=2, gated=True)
    args["x"][M // 2, 17] = float("nan")
    args["Wt"][5, 3] = float("inf")
    nmm.nmm_gemv_nt_act(args["x"], args["Wt"], y, K=K, act=2, gated=True)
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[M // 2], keep[:, 5] = False, False
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[M // 2]).all()


def test_no_products_in_tiles_leave_the_epilogue():
    r = torch.randn((400, 5000), device="cuda").to(torch.float16)
    x, Wt = torch.zeros((400, 8), dtype=torch.float16, device="cuda"), torch.zeros((5000, 8), dtype=torch.float16, device="cuda")
    y = torch.zeros_like(r)
    nmm.nmm_gemv_nt_act(x, Wt, y, K=0, residual=r)
    assert torch.equal(y, r)
