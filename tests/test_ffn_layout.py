"""CPU models of the address arithmetic of nt_rows.h and nt_wide.h: what a workgroup's loads put into LDS is what its waves read, every
access lies inside its array, every (row of x, row of the weight) pair of a tile is one lane's, and the walk over the items of a
launch visits each once."""
import numpy as np
import pytest

ROW = 128                 # bytes of a row in a slot of 64 k
TILE = 16 * ROW


@pytest.mark.parametrize("BM,BN,S", [(64, 128, 3), (128, 128, 3), (256, 128, 3)])
def test_wide_tiles(BM, BN, S):
    waves = 8
    NT = 4 if BM >= 256 else 2
    WN = BN // 16 // NT
    WM = waves // WN
    MT, LW = BM // WM // 16, BN // 64
    slot = (BM + BN) * ROW
    assert WM * WN == waves and MT * WM * 16 == BM and S * slot + 4 * 1025 + 64 <= 160 * 1024
    lds = np.full((slot // 16, 2), -1)                     # the (row, chunk) of each 16 bytes
    lane = np.arange(64)
    for wave in range(waves):
        chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)
        for i in range(LW + BM // 64):
            r = 8 * (wave + waves * i) + (lane >> 3)       # past BN: rows of x
            at = (8 * wave * ROW + 64 * i * ROW) // 16 + lane
            assert (lds[at] == -1).all() and at.max() < slot // 16
            assert ((r < BN) == (i < LW)).all()
            lds[at] = np.stack((r, chunk), 1)
    assert (lds >= 0).all()
    g, j = lane >> 4, lane & 15
    f0 = j * ROW + ((g ^ (j >> 1)) << 4)
    seen = np.zeros((BM, BN), dtype=int)
    for wave in range(waves):
        wm, wn = wave % WM, wave // WM
        wa, xa = f0 + wn * NT * TILE, f0 + BN * ROW + wm * TILE
        for h in (0, 1):
            for t in range(NT):
                got = lds[((wa ^ (64 * h)) + t * TILE) // 16]
                assert (got[:, 0] == (wn * NT + t) * 16 + j).all() and (got[:, 1] == 4 * h + g).all()
            for m in range(MT):
                got = lds[((xa ^ (64 * h)) + m * WM * TILE) // 16]
                assert (got[:, 0] == BN + (wm + WM * m) * 16 + j).all() and (got[:, 1] == 4 * h + g).all()
        for t in range(NT):
            for m in range(MT):
                for i in range(4):
                    seen[(wm + WM * m) * 16 + j, (wn * NT + t) * 16 + 4 * g + i] += 1
    assert (seen == 1).all()
    # fewer rows than BM: the loads and tiles that are run cover them
    for mrows in range(1, BM + 1):
        M = next(u for u in range(1, MT + 1) if u == MT or mrows <= 16 * WM * u)
        assert 16 * WM * M >= mrows and 64 * ((16 * WM * M + 63) // 64) >= 16 * WM * M
    # the sums, [m][row of the weight] with 4 floats of padding, in the ring's place
    assert BM * (BN + 4) * 4 <= S * slot
    # a fragment's 16 rows lie in 16 different 16-byte places of LDS's 256-byte lines
    for q in range(4):
        assert len(set((f0[16 * q:16 * q + 16] // 16) % 16)) == 16


@pytest.mark.parametrize("BN,WN", [(128, 4), (128, 2)])
def test_rows_of_a_gated_weight_in_a_wide_tile(BN, WN):
    """Gate and up rows of one output column lie half a wave's rows apart; every column of the block once."""
    wave_rows, N, n0 = BN // WN, 10 ** 6, 640
    r = np.arange(BN)
    rr = r % wave_rows
    n = n0 + r // wave_rows * (wave_rows // 2) + rr % (wave_rows // 2)
    up = rr >= wave_rows // 2
    place = {(int(a), bool(b)): int(c) for a, b, c in zip(n, up, r)}
    assert len(place) == BN
    for c in range(0, BN // 2, 4):
        at = c // (wave_rows // 2) * wave_rows + c % (wave_rows // 2)
        for i in range(4):
            assert place[(n0 + c + i, False)] == at + i and place[(n0 + c + i, True)] == at + i + wave_rows // 2


@pytest.mark.parametrize("n_blocks", [1, 2, 7, 8, 9, 56, 57])
@pytest.mark.parametrize("ks", [1, 2, 4, 8])
def test_every_item_once(n_blocks, ks):
    """Dense: (block of columns, row tile, slice of K) over XCDs and workgroups; grouped (ks 1): experts with 0 to 3 tiles."""
    share = 8 // ks
    nbx = -(-n_blocks // share)
    for tiles in ([1], [3], [0, 2, 0, 1, 3, 0], [0]):
        if ks > 1 and len(tiles) > 1:
            continue
        starts = np.concatenate(([0], np.cumsum(tiles)))
        seen = {}
        for grid in (8, 64):
            seen.clear()
            for bid in range(grid):
                xcd, slice_ = bid & 7, (bid & 7) % ks
                for idx in range(bid >> 3, int(starts[-1]) * nbx, grid >> 3):
                    u = idx // nbx
                    e = int(np.searchsorted(starts, u, side="right")) - 1
                    rem = idx - int(starts[e]) * nbx
                    nbi, rt = rem // tiles[e], rem % tiles[e]
                    nb = share * nbi + xcd // ks
                    if nb < n_blocks:
                        seen[(e, rt, nb, slice_)] = seen.get((e, rt, nb, slice_), 0) + 1
            want = {(e, rt, nb, s) for e, n in enumerate(tiles) for rt in range(n) for nb in range(n_blocks) for s in range(ks)}
            assert set(seen) == want and all(v == 1 for v in seen.values())


@pytest.mark.parametrize("XR,NT", [(1, 1), (1, 2), (2, 2), (4, 1), (4, 2), (8, 2)])
def test_few_rows(XR, NT):
    """rows_kernel's ring: loads of 4 rows x 256 bytes, chunk c of row r at place c ^ (r % 16), fragments of 16 rows."""
    lane = np.arange(64)
    g, j = lane >> 4, lane & 15
    loads = 4 * NT + XR
    lds = np.full((loads * 64, 2), -1)
    for q in range(loads):
        r = 4 * (q if q < 4 * NT else q - 4 * NT) + g
        lds[q * 64 + lane] = np.stack((r, j ^ (r & 15)), 1)
    wa = j * 256 + ((g ^ j) * 16)
    jx = j & (4 * XR - 1) if XR < 4 else j
    xa = jx * 256 + ((g ^ jx) * 16)
    for step in range(4):
        for t in range(NT):
            got = lds[(4096 * t + (wa ^ (64 * step))) // 16]
            assert (got[:, 0] == 16 * t + j).all() and (got[:, 1] == 4 * step + g).all()
        for t in range(2 if XR > 4 else 1):
            at = (4 * NT * 1024 + 4096 * t + (xa ^ (64 * step))) // 16
            assert at.max() < loads * 64
            got = lds[at]
            assert (got[:, 0] == 16 * t + jx).all() and (got[:, 1] == 4 * step + g).all()
