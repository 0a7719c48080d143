"""nmm_gemv_w4 against the product with the weight that its codes stand for, in 64 bits.

Integer inputs and power-of-two scales make every partial sum exact, so those results must be equal.  For other
inputs the bound is derived: products are exact; a group's sum passes at most 8 MFMAs of 32 products, the two sums
of an integer group meet in one fused operation, then K / 32 groups, 4 waves and the slices are added, each of
these at most one ulp (2^-23) of the sum of magnitudes sum_k |x_k| s (code + zero).
"""
import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

nmm = pytest.importorskip("paper_2609_16009_amd")


def make(seed, M, K, N, group, mx, zeros, fp16, integer, pad=0):
    rng = np.random.default_rng(seed)
    dt = torch.float16 if fp16 else torch.bfloat16
    ldx, ldw, groups = (K + 7) // 8 * 8 + 8 * pad, (K + 31) // 32 * 16 + 16 * pad, -(-K // group)
    x = np.full((M, ldx), np.nan)                      # past K: NaN that may not reach a result
    x[:, :K] = rng.integers(-4, 5, (M, K)) if integer else rng.standard_normal((M, K))
    xt = torch.from_numpy(x.astype(np.float32)).to(dt)
    x = xt[:, :K].double().numpy()
    codes = rng.integers(0, 256, (N, ldw), dtype=np.uint8)
    if mx:
        scales = rng.integers(125, 130, (N, groups), dtype=np.uint8)
        st, z = torch.from_numpy(scales), None
    else:
        scales = 2.0 ** rng.integers(-2, 3, (N, groups)) if integer else rng.uniform(0.002, 0.02, (N, groups))
        st = torch.from_numpy(scales.astype(np.float32)).to(dt)
        scales = st.double().numpy()
        z = rng.integers(0, 16, (N, groups), dtype=np.uint8) if zeros else None
    if pad:                                            # padded rows of scales and zeros too
        st = torch.nn.functional.pad(st, (0, pad + 2))
    W = ob.w4_decode(codes, scales, group, K, z, mx)
    mag = np.abs(W) if mx or integer else np.abs(W) + 2 * np.abs(ob.w4_decode(np.zeros_like(codes), scales, group, K, z))
    args = dict(x=xt.cuda(), Wq=torch.from_numpy(codes).cuda(), scales=st.cuda(), group=group, K=K,
                zeros=None if z is None else torch.from_numpy(z).cuda())
    return args, x @ W.T, np.abs(x) @ mag.T


def run(args, M, N, **kw):
    y = torch.full((M, N + 3), float("nan"), device="cuda")
    nmm.nmm_gemv_w4(y=y, **args, **kw)
    return y


def check(seed, M, K, N, group, mx=False, zeros=False, fp16=False, integer=True, pad=0, what=""):
    args, ref, mag = make(seed, M, K, N, group, mx, zeros, fp16, integer, pad)
    y = run(args, M, N).double().cpu().numpy()
    assert np.isnan(y[:, N:]).all(), "columns past N"
    y = y[:, :N]
    if integer:
        bad = y != ref
    else:
        bad = ~(np.abs(y - ref) <= (8 * 33 + 1 + K / 32 + 4 + 64) * 2.0 ** -23 * mag)
    assert not bad.any(), f"{what or (M, K, N, group, mx, zeros, fp16)}: {bad.sum()} of {bad.size} wrong, first " \
                          f"{np.argwhere(bad)[0]}: {y[bad][0]} for {ref[bad][0]}"


KINDS = [(32, True, False), (32, False, False), (32, False, True), (64, False, True), (128, False, False),
         (256, False, True), (1024, False, False)]


@pytest.mark.parametrize("fp16", [False, True], ids=["bf16", "f16"])
@pytest.mark.parametrize("group,mx,zeros", KINDS)
def test_integers_exact_at_every_row_count(group, mx, zeros, fp16):
    for M in (1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 70):
        check(M + group, M, 777, 100, group, mx, zeros, fp16)


@pytest.mark.parametrize("M", [1, 8, 32])
@pytest.mark.parametrize("group,mx,zeros", KINDS)
@pytest.mark.parametrize("K,N", [(1, 1), (7, 17), (31, 15), (32, 16), (33, 5), (255, 33), (256, 64), (257, 1), (1024, 130),
                                 (2049, 31), (4099, 203), (9000, 16), (16384, 48)])
def test_integers_exact_at_odd_sizes(K, N, group, mx, zeros, M):
    check(K + N + M, M, K, N, group, mx, zeros)


@pytest.mark.parametrize("fp16", [False, True], ids=["bf16", "f16"])
@pytest.mark.parametrize("mx", [False, True], ids=["int", "mx"])
def test_every_code_and_zero(mx, fp16):
    # one weight a row against x = 1: each code under each zero point
    codes = np.zeros((256, 16), dtype=np.uint8)
    codes[:, 0] = np.tile(np.arange(16), 16)
    dt = torch.float16 if fp16 else torch.bfloat16
    x = torch.zeros((1, 32), dtype=dt, device="cuda")
    x[0, 0] = 1
    zeros = np.repeat(np.arange(16), 16).astype(np.uint8)[:, None] * 17           # 0 .. 255
    scales = np.full((256, 1), 127, np.uint8) if mx else np.ones((256, 1))
    st = torch.from_numpy(scales).cuda() if mx else torch.ones((256, 1), dtype=dt, device="cuda")
    y = torch.zeros((1, 256), device="cuda")
    nmm.nmm_gemv_w4(x, torch.from_numpy(codes).cuda(), st, y, group=32, zeros=None if mx else torch.from_numpy(zeros).cuda())
    W = ob.w4_decode(codes, scales, 32, 32, None if mx else zeros, mx)
    assert np.array_equal(y.cpu().numpy()[0], W[:, 0])


def test_power_of_two_scales_over_their_range():
    b = np.arange(256, dtype=np.uint8)[:, None]
    codes = np.zeros((256, 16), dtype=np.uint8)
    codes[:, 0] = 2                                                                # 1.0
    x = torch.zeros((1, 32), dtype=torch.bfloat16, device="cuda")
    x[0, 0] = 1
    y = torch.zeros((1, 256), device="cuda")
    nmm.nmm_gemv_w4(x, torch.from_numpy(codes).cuda(), torch.from_numpy(b).cuda(), y, group=32)
    got = y.cpu().numpy()[0].astype(np.float64)
    assert np.array_equal(got[1:255], np.exp2(np.arange(1, 255) - 127.0))
    assert got[0] in (0.0, 2.0 ** -127) and np.isnan(got[255])                     # a subnormal may be flushed


@pytest.mark.parametrize("M,K,N,group,mx,zeros,fp16", [
    (1, 16384, 512, 128, False, False, False), (8, 1536, 2048, 32, True, False, False),
    (5, 4099, 5003, 64, False, True, True), (32, 7168, 576, 128, False, True, False), (3, 16384, 100, 32, True, False, True)])
def test_real_values(M, K, N, group, mx, zeros, fp16):
    check(K, M, K, N, group, mx, zeros, fp16, integer=False)


def test_padded_rows():
    for M in (1, 6, 20):
        check(M, M, 1000, 90, 64, False, False, pad=3)
        check(M, M, 1000, 90, 32, True, False, pad=2)


def test_random_shapes():
    rng = np.random.default_rng(5)
    for k in range(40):
        group, mx, zeros = KINDS[int(rng.integers(len(KINDS)))]
        M, K, N = int(rng.integers(1, 40)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 11))
        print(f"case {k}: {M} x {K} x {N}, group {group}, mx {mx}, zeros {zeros}", flush=True)
        check(200 + k, M, K, N, group, mx, zeros, fp16=bool(rng.integers(2)))


def test_empty_problems():
    w, s = torch.zeros((4, 16), dtype=torch.uint8, device="cuda"), torch.ones((4, 1), dtype=torch.bfloat16, device="cuda")
    x = torch.ones((2, 32), dtype=torch.bfloat16, device="cuda")
    y = torch.full((2, 4), 5.0, device="cuda")
    nmm.nmm_gemv_w4(x[:0], w, s, y, group=32)
    nmm.nmm_gemv_w4(x, w[:0], s[:0], y, group=32)
    assert bool((y == 5.0).all())
    nmm.nmm_gemv_w4(x, w, s, y, group=32, K=0)
    assert bool((y == 0.0).all())


def test_streams_captured_replays_and_the_same_bits():
    args, _, _ = make(3, 4, 16384, 96, 32, False, True, False, integer=False)      # K split over workgroups
    assert nmm.lib().nmm_gemv_w4_workspace_size(4, 16384, 96, 32) > 0
    want = run(args, 4, 96)
    torch.cuda.synchronize()
    for _ in range(5):
        assert torch.equal(run(args, 4, 96)[:, :96], want[:, :96])
    ws, y = nmm.Workspace(), torch.zeros((4, 96), device="cuda")
    nmm.nmm_gemv_w4(y=y, workspace=ws, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nmm.nmm_gemv_w4(y=y, workspace=ws, **args)
    for _ in range(3):
        args["x"][:, :16384].normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, run(args, 4, 96)[:, :96])
    side = torch.cuda.Stream()
    other = run(args, 4, 96, stream=side)
    side.synchronize()
    assert torch.equal(other[:, :96], y)


@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 9, 16, 17, 33])
@pytest.mark.parametrize("group,mx,zeros", [(32, True, False), (32, False, True), (128, False, True), (512, False, False)])
def test_every_end_of_a_slot(M, group, mx, zeros):
    for K in (225, 255, 256, 257, 1023, 1032, 1281, 2311, 4095):       # slots of 256, four of them in flight
        check(M * K, M, K, 70, group, mx, zeros, fp16=K % 2 == 0)


@pytest.mark.parametrize("M", [1, 8, 12, 32])
def test_many_slices_and_slots(M):
    check(M, M, 40000, 130, 32, False, True)                           # K-slices as long as their scales allow
    check(M, M, 40000, 130, 32, True, False)
    check(M, M, 60001, 65, 4096, False, True)                          # groups longer than a slice


def test_more_row_blocks_than_counters():
    M, K, N = 130, 544, 1 << 19                                        # 128 rows a launch
    rng = np.random.default_rng(9)
    x = torch.from_numpy(rng.integers(-4, 5, (M, K)).astype(np.float32)).to(torch.bfloat16).cuda()
    codes = torch.randint(0, 256, (N, 272), dtype=torch.uint8, device="cuda")
    scales = (2.0 ** torch.randint(-2, 3, (N, 17), device="cuda")).to(torch.bfloat16)
    y = torch.full((M, N), float("nan"), device="cuda")
    nmm.nmm_gemv_w4(x, codes, scales, y, group=32)
    at = torch.cat((torch.arange(0, N, 4097, device="cuda"), torch.tensor([N - 1], device="cuda")))
    W = ob.w4_decode(codes[at].cpu().numpy(), scales[at].double().cpu().numpy(), 32, K)
    assert np.array_equal(y[:, at].double().cpu().numpy(), x.double().cpu().numpy() @ W.T)
    assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("M", [4, 20])
@pytest.mark.parametrize("mx", [False, True])
def test_what_is_not_finite_stays_in_its_row(M, mx):
    args, ref, _ = make(17, M, 700, 96, 32, mx, not mx, False, True)
    args["x"][1, 300] = float("inf")
    args["x"][2, 5] = float("nan")
    if mx:
        args["scales"][7, 3] = 255
    else:
        args["scales"][7, 3] = float("nan")
    y = run(args, M, 96)[:, :96].double().cpu().numpy()
    assert not np.isfinite(y[1]).any()
    assert np.isnan(y[2]).all() and np.isnan(y[:, 7]).all()
    rows, cols = np.delete(np.arange(M), [1, 2]), np.delete(np.arange(96), 7)
    assert np.array_equal(y[np.ix_(rows, cols)], ref[np.ix_(rows, cols)])


def test_two_streams_with_their_own_workspaces():
    args, _, _ = make(3, 4, 16384, 96, 32, False, True, False, integer=False)
    other, _, _ = make(4, 24, 8192, 200, 128, False, False, False, integer=False)
    want = run(args, 4, 96)[:, :96].clone(), run(other, 24, 200)[:, :200].clone()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        y1, y2 = torch.zeros((4, 96), device="cuda"), torch.zeros((24, 200), device="cuda")
        torch.cuda.synchronize()
        nmm.nmm_gemv_w4(y=y1, stream=s1, **args)
        nmm.nmm_gemv_w4(y=y2, stream=s2, **other)
        torch.cuda.synchronize()
        assert torch.equal(y1, want[0]) and torch.equal(y2, want[1])


def test_python_refusals():
    x = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda")
    w, s, y = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros_like(x[:1, :2]).repeat(8, 1), torch.zeros((2, 8), device="cuda")
    z = torch.zeros((8, 2), dtype=torch.uint8, device="cuda")
    nmm.nmm_gemv_w4(x, w, s, y, group=32, zeros=z)
    for bad in (dict(x=x.float()), dict(Wq=w.to(torch.int8)), dict(y=y.bfloat16()), dict(scales=s.float()), dict(scales=s.half()),
                dict(zeros=z.to(torch.int8))):
        with pytest.raises(TypeError):
            nmm.nmm_gemv_w4(**{**dict(x=x, Wq=w, scales=s, y=y, group=32, zeros=z), **bad})
    for bad in (dict(x=x.cpu()), dict(y=y[:1]), dict(y=y[:, :7]), dict(scales=s[:7]), dict(scales=s[:, :1]), dict(zeros=z[:7]),
                dict(zeros=z[:, :1]), dict(K=65), dict(Wq=w[:, :16]), dict(group=48), dict(group=0), dict(K=-1),
                dict(scales=z), dict(x=x[0]), dict(Wq=w[0]), dict(y=y[0]), dict(scales=s[:, 0]), dict(x=x.t())):
        with pytest.raises((ValueError, nmm.NmmError)):                 # the binding's checks, the library's
            nmm.nmm_gemv_w4(**{**dict(x=x, Wq=w, scales=s, y=y, group=32, zeros=z), **bad})
