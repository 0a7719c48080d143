"""The feed-forward operators' entry points without a GPU: every invalid argument is refused before the device is touched."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import ffn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
nmm = pytest.importorskip("paper_2609_16009_amd")
if not os.path.exists(nmm.LIB_PATH):
    pytest.skip("libnmm.so not built", allow_module_level=True)

L = nmm.lib()
A = 1 << 30          # a fake, 256-byte aligned "device address"; never dereferenced here
FAR = 1 << 40        # another, far behind it
LIM = 1 << 31


def fill(struct, defaults, kw):
    assert set(kw) <= set(defaults)
    for k, v in {**defaults, **kw}.items():
        setattr(struct, k, v)
    return struct


def act_of(**kw):
    return fill(nmm.nmm_nt_act(), dict(M=4, K=512, N=256, dt=nmm.NMM_BF16, act=nmm.NMM_ACT_SILU, gated=0, x=A, ldx=512, Wt=2 * A,
                                       ldwt=512, bias=3 * A, residual=4 * A, ldr=256, y=5 * A, ldy=256, y_f32=6 * A, ldyf=256), kw)


def run_act(**kw):
    return L.nmm_gemv_nt_act(ctypes.byref(act_of(**kw)), None, 0, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=0), nmm.NMM_ERR_DTYPE), (dict(dt=3), nmm.NMM_ERR_DTYPE), (dict(act=-1), nmm.NMM_ERR_ARG), (dict(act=5), nmm.NMM_ERR_ARG),
    (dict(gated=2), nmm.NMM_ERR_ARG), (dict(gated=-1), nmm.NMM_ERR_ARG),
    (dict(M=-1), nmm.NMM_ERR_SHAPE), (dict(K=-1), nmm.NMM_ERR_SHAPE), (dict(N=-1), nmm.NMM_ERR_SHAPE),
    (dict(M=LIM), nmm.NMM_ERR_SHAPE), (dict(K=LIM), nmm.NMM_ERR_SHAPE), (dict(N=LIM), nmm.NMM_ERR_SHAPE),
    (dict(ldx=504), nmm.NMM_ERR_SHAPE), (dict(ldwt=504), nmm.NMM_ERR_SHAPE), (dict(ldr=255), nmm.NMM_ERR_SHAPE),
    (dict(ldy=255), nmm.NMM_ERR_SHAPE), (dict(ldyf=255), nmm.NMM_ERR_SHAPE), (dict(ldx=LIM), nmm.NMM_ERR_SHAPE),
    (dict(ldwt=LIM), nmm.NMM_ERR_SHAPE), (dict(ldr=LIM), nmm.NMM_ERR_SHAPE), (dict(ldy=LIM), nmm.NMM_ERR_SHAPE),
    (dict(ldyf=LIM), nmm.NMM_ERR_SHAPE),
    (dict(N=1 << 21, ldy=1 << 21, ldr=1 << 21, ldyf=1 << 21), nmm.NMM_ERR_SHAPE),                  # a weight of 2^31 bytes
    (dict(N=1 << 20, ldy=1 << 20, ldr=1 << 20, ldyf=1 << 20, gated=1), nmm.NMM_ERR_SHAPE),         # and a gated one
    (dict(K=0, N=1 << 30, ldy=1 << 30, ldr=1 << 30, ldyf=1 << 30), nmm.NMM_ERR_SHAPE),
    (dict(M=2, ldx=1 << 30), nmm.NMM_ERR_SHAPE), (dict(M=128, ldx=1 << 24), nmm.NMM_ERR_SHAPE),    # a block of x past 2^31 bytes
    (dict(ldx=516), nmm.NMM_ERR_ALIGN), (dict(ldwt=516), nmm.NMM_ERR_ALIGN), (dict(x=A + 8), nmm.NMM_ERR_ALIGN),
    (dict(Wt=A + 8), nmm.NMM_ERR_ALIGN), (dict(bias=A + 1), nmm.NMM_ERR_ALIGN), (dict(residual=A + 1), nmm.NMM_ERR_ALIGN),
    (dict(y=A + 1), nmm.NMM_ERR_ALIGN), (dict(y_f32=A + 2), nmm.NMM_ERR_ALIGN),
    (dict(x=None), nmm.NMM_ERR_NULL), (dict(Wt=None), nmm.NMM_ERR_NULL), (dict(y=None, y_f32=None), nmm.NMM_ERR_NULL),
    # outputs over what is read, and over each other
    (dict(residual=5 * A + 2), nmm.NMM_ERR_ARG), (dict(residual=5 * A, ldr=264), nmm.NMM_ERR_ARG),
    (dict(residual=6 * A), nmm.NMM_ERR_ARG), (dict(y=6 * A + 512), nmm.NMM_ERR_ARG), (dict(y=A), nmm.NMM_ERR_ARG),
    (dict(y_f32=A), nmm.NMM_ERR_ARG), (dict(y=A + 1000, ldy=512), nmm.NMM_ERR_ARG), (dict(y=A + 512, ldx=760, ldy=760), nmm.NMM_ERR_ARG),
])
def test_product_refuses(kw, status):
    assert run_act(**kw) == status


def test_product_of_nothing():
    assert run_act(M=0, x=None, Wt=None, y=None, y_f32=None) == nmm.NMM_OK
    assert run_act(N=0, y=None, y_f32=None) == nmm.NMM_OK
    assert L.nmm_gemv_nt_act(None, None, 0, None) == nmm.NMM_ERR_NULL
    assert L.nmm_gemv_nt_act_workspace_size(None) == 0
    assert L.nmm_gemv_nt_act_workspace_size(ctypes.byref(act_of(M=-1))) == 0


def router_of(**kw):
    return fill(nmm.nmm_moe_router(), dict(tokens=64, experts=256, top_k=8, logits=A, logits_type=nmm.NMM_SRC_F32, ld_logits=256,
                                           score=nmm.NMM_SCORE_SIGMOID, bias=A, groups=8, top_groups=4, group_top=2, renormalize=1,
                                           scale=2.5, mask=A, chosen=A, weights=A, offsets=A, pairs=A), kw)


@pytest.mark.parametrize("kw,status", [
    (dict(logits_type=2), nmm.NMM_ERR_DTYPE), (dict(tokens=-1), nmm.NMM_ERR_SHAPE), (dict(tokens=1 << 26, top_k=1), nmm.NMM_ERR_SHAPE),
    (dict(tokens=1 << 23), nmm.NMM_ERR_SHAPE), (dict(tokens=1 << 62, top_k=4), nmm.NMM_ERR_SHAPE), (dict(experts=0), nmm.NMM_ERR_SHAPE),
    (dict(experts=1025, groups=1, top_groups=1, ld_logits=1025), nmm.NMM_ERR_SHAPE), (dict(experts=-8), nmm.NMM_ERR_SHAPE),
    (dict(top_k=0), nmm.NMM_ERR_SHAPE), (dict(top_k=33), nmm.NMM_ERR_SHAPE), (dict(groups=0), nmm.NMM_ERR_SHAPE),
    (dict(groups=7), nmm.NMM_ERR_SHAPE), (dict(groups=128), nmm.NMM_ERR_SHAPE), (dict(top_groups=0), nmm.NMM_ERR_SHAPE),
    (dict(top_groups=9), nmm.NMM_ERR_SHAPE), (dict(groups=64, top_groups=1), nmm.NMM_ERR_SHAPE),      # 8 of 4 experts
    (dict(ld_logits=255), nmm.NMM_ERR_SHAPE), (dict(ld_logits=LIM), nmm.NMM_ERR_SHAPE),
    (dict(score=0), nmm.NMM_ERR_ARG), (dict(score=3), nmm.NMM_ERR_ARG), (dict(group_top=0), nmm.NMM_ERR_ARG),
    (dict(group_top=3), nmm.NMM_ERR_ARG), (dict(renormalize=2), nmm.NMM_ERR_ARG), (dict(scale=float("nan")), nmm.NMM_ERR_ARG),
    (dict(scale=float("inf")), nmm.NMM_ERR_ARG),
    (dict(logits=None), nmm.NMM_ERR_NULL), (dict(chosen=None), nmm.NMM_ERR_NULL), (dict(weights=None), nmm.NMM_ERR_NULL),
    (dict(offsets=None), nmm.NMM_ERR_NULL), (dict(pairs=None), nmm.NMM_ERR_NULL), (dict(tokens=0, offsets=None), nmm.NMM_ERR_NULL),
    (dict(logits=A + 2), nmm.NMM_ERR_ALIGN), (dict(logits=A + 1, logits_type=nmm.NMM_SRC_BF16), nmm.NMM_ERR_ALIGN),
    (dict(bias=A + 2), nmm.NMM_ERR_ALIGN), (dict(chosen=A + 2), nmm.NMM_ERR_ALIGN), (dict(weights=A + 1), nmm.NMM_ERR_ALIGN),
    (dict(offsets=A + 2), nmm.NMM_ERR_ALIGN), (dict(pairs=A + 2), nmm.NMM_ERR_ALIGN),
    (dict(), nmm.NMM_ERR_WORKSPACE),
])
def test_route_refuses(kw, status):
    assert L.nmm_moe_route(ctypes.byref(router_of(**kw)), None, 0, None) == status


def test_route_workspace():
    assert L.nmm_moe_route(None, None, 0, None) == nmm.NMM_ERR_NULL
    size = lambda **kw: L.nmm_moe_route_workspace_size(ctypes.byref(router_of(**kw)))
    assert L.nmm_moe_route_workspace_size(None) == 0 and size(tokens=-1) == 0 and size(experts=0) == 0 and size(tokens=0) == 0
    assert size(tokens=64) == 65536
    for tokens, experts, k in ((4097, 256, 8), (32768, 64, 6), ((1 << 23) - 1, 1024, 8), ((1 << 26) - 1, 8, 1)):
        segments, rest = divmod(size(tokens=tokens, experts=experts, top_k=k, groups=1, top_groups=1) - 65536, 4 * experts)
        assert rest == 0 and segments >= 1


def ffn_of(**kw):
    d = dict(tokens=16, top_k=4, experts=32, first=8, local=8, hidden=512, inner=256, dt=nmm.NMM_BF16, act=nmm.NMM_ACT_SILU, x=A,
             ldx=512, W1=FAR, ldw1=512, stride1=512 * 512, W2=2 * FAR, ldw2=256, stride2=512 * 256, chosen=A, weights=A, offsets=A,
             pairs=A, residual=2 * A, ldr=512, y=3 * A, ldy=512)
    return fill(nmm.nmm_moe_ffn(), d, kw)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=0), nmm.NMM_ERR_DTYPE), (dict(act=5), nmm.NMM_ERR_ARG), (dict(act=-1), nmm.NMM_ERR_ARG),
    (dict(tokens=-1), nmm.NMM_ERR_SHAPE), (dict(tokens=1 << 24), nmm.NMM_ERR_SHAPE), (dict(tokens=1 << 62), nmm.NMM_ERR_SHAPE),
    (dict(top_k=0), nmm.NMM_ERR_SHAPE), (dict(top_k=33), nmm.NMM_ERR_SHAPE), (dict(experts=0), nmm.NMM_ERR_SHAPE),
    (dict(experts=1025), nmm.NMM_ERR_SHAPE), (dict(first=-1), nmm.NMM_ERR_SHAPE), (dict(local=-1), nmm.NMM_ERR_SHAPE),
    (dict(first=25), nmm.NMM_ERR_SHAPE), (dict(local=25), nmm.NMM_ERR_SHAPE), (dict(hidden=0), nmm.NMM_ERR_SHAPE),
    (dict(inner=0), nmm.NMM_ERR_SHAPE), (dict(hidden=-1), nmm.NMM_ERR_SHAPE), (dict(inner=1 << 30), nmm.NMM_ERR_SHAPE),
    (dict(ldx=504), nmm.NMM_ERR_SHAPE), (dict(ldw1=504), nmm.NMM_ERR_SHAPE), (dict(ldw2=248), nmm.NMM_ERR_SHAPE),
    (dict(ldy=511), nmm.NMM_ERR_SHAPE), (dict(ldr=511), nmm.NMM_ERR_SHAPE), (dict(ldx=LIM), nmm.NMM_ERR_SHAPE),
    (dict(ldw1=1 << 22), nmm.NMM_ERR_SHAPE), (dict(ldw2=1 << 22), nmm.NMM_ERR_SHAPE),          # an expert of 2^31 bytes
    (dict(stride1=512 * 512 - 8), nmm.NMM_ERR_SHAPE), (dict(stride2=512 * 256 - 8), nmm.NMM_ERR_SHAPE),
    (dict(stride1=1 << 50), nmm.NMM_ERR_SHAPE), (dict(stride2=1 << 50), nmm.NMM_ERR_SHAPE),
    (dict(tokens=(1 << 20) + 1, ldx=1 << 10), nmm.NMM_ERR_SHAPE),                                # x of 2^31 bytes
    (dict(ldx=516), nmm.NMM_ERR_ALIGN), (dict(ldw1=516, stride1=1 << 20), nmm.NMM_ERR_ALIGN), (dict(ldw2=260, stride2=1 << 20), nmm.NMM_ERR_ALIGN),
    (dict(stride1=(1 << 20) + 4), nmm.NMM_ERR_ALIGN), (dict(stride2=(1 << 20) + 4), nmm.NMM_ERR_ALIGN),
    (dict(x=A + 8), nmm.NMM_ERR_ALIGN), (dict(W1=A + 8), nmm.NMM_ERR_ALIGN), (dict(W2=A + 8), nmm.NMM_ERR_ALIGN),
    (dict(y=3 * A + 1), nmm.NMM_ERR_ALIGN), (dict(residual=2 * A + 1), nmm.NMM_ERR_ALIGN), (dict(chosen=A + 2), nmm.NMM_ERR_ALIGN),
    (dict(weights=A + 2), nmm.NMM_ERR_ALIGN), (dict(offsets=A + 2), nmm.NMM_ERR_ALIGN), (dict(pairs=A + 2), nmm.NMM_ERR_ALIGN),
    (dict(x=None), nmm.NMM_ERR_NULL), (dict(W1=None), nmm.NMM_ERR_NULL), (dict(W2=None), nmm.NMM_ERR_NULL),
    (dict(y=None), nmm.NMM_ERR_NULL), (dict(chosen=None), nmm.NMM_ERR_NULL), (dict(weights=None), nmm.NMM_ERR_NULL),
    (dict(offsets=None), nmm.NMM_ERR_NULL), (dict(pairs=None), nmm.NMM_ERR_NULL),
    (dict(y=A), nmm.NMM_ERR_ARG), (dict(y=2 * A + 2), nmm.NMM_ERR_ARG), (dict(residual=3 * A, ldr=520), nmm.NMM_ERR_ARG),
    (dict(), nmm.NMM_ERR_WORKSPACE), (dict(residual=3 * A), nmm.NMM_ERR_WORKSPACE),              # in place is allowed
    # column ranges of one buffer that take turns
    (dict(x=A, ldx=1024, y=A + 1024, ldy=1024), nmm.NMM_ERR_WORKSPACE), (dict(x=A, ldx=1024, y=A + 1022, ldy=1024), nmm.NMM_ERR_ARG),
    (dict(x=A + 1024, ldx=1024, y=A, ldy=1024), nmm.NMM_ERR_WORKSPACE), (dict(x=A + 1024, ldx=1016, y=A, ldy=1016), nmm.NMM_ERR_ARG),
])
def test_experts_refuse(kw, status):
    assert L.nmm_moe_experts(ctypes.byref(ffn_of(**kw)), None, 0, None) == status


def test_experts_of_nothing_and_workspace():
    assert L.nmm_moe_experts(ctypes.byref(ffn_of(tokens=0, x=None, y=None)), None, 0, None) == nmm.NMM_OK
    assert L.nmm_moe_experts(None, None, 0, None) == nmm.NMM_ERR_NULL
    size = lambda **kw: L.nmm_moe_experts_workspace_size(ctypes.byref(ffn_of(**kw)))
    assert L.nmm_moe_experts_workspace_size(None) == 0
    assert size(tokens=-1) == size(tokens=0) == size(local=0) == size(hidden=0) == size(experts=0) == 0
    for tokens, k, hidden, inner in ((1, 8, 7168, 2048), (64, 8, 7168, 2048), (37, 3, 1037, 331), (1, 1, 1, 1)):
        need = 65536 + tokens * k * (2 * inner + 4 * hidden)
        assert need <= size(tokens=tokens, top_k=k, hidden=hidden, inner=inner) <= need + tokens * k * 144 + 256


STRUCTS = {"nmm_nt_act": act_of, "nmm_moe_router": router_of, "nmm_moe_ffn": ffn_of}


def test_struct_layouts_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "nmm.h"', "int main(void) {"]
    for st in STRUCTS:
        lines.append(f'  printf("{st} sizeof %zu\\n", sizeof({st}));')
        lines += [f'  printf("{st} {f} %zu\\n", offsetof({st}, {f}));' for f, _ in getattr(nmm, st)._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = {tuple(l.split()[:2]): int(l.split()[2]) for l in subprocess.run([str(exe)], capture_output=True, text=True,
                                                                           check=True).stdout.split("\n") if l}
    for st in STRUCTS:
        cls = getattr(nmm, st)
        assert got[(st, "sizeof")] == ctypes.sizeof(cls), st
        for f, _ in cls._fields_:
            assert got[(st, f)] == getattr(cls, f).offset, (st, f)


@pytest.mark.parametrize("st,packed", [("nmm_nt_act", "_NT_ACT"), ("nmm_moe_router", "_ROUTER"), ("nmm_moe_ffn", "_FFN")])
def test_packed_arguments_match_the_structs(st, packed):
    cls = getattr(nmm, st)
    values = [0.5 if t is ctypes.c_float else 3 + 2 * i for i, (_, t) in enumerate(cls._fields_)]
    s = cls(*values)
    assert getattr(nmm, packed).pack(*values) == bytes(s)


def test_the_oracle_of_the_route():
    """By hand: two groups of two, the second one's two best win; ties to the lowest index; a padded token."""
    logits = np.log(np.array([[0.3, 0.1, 0.25, 0.35], [0.25, 0.25, 0.25, 0.25], [0.4, 0.3, 0.2, 0.1]]))
    chosen, w, offsets, pairs = ffn.route(logits, 2, True, groups=2, top_groups=1, group_top=2, mask=[1, 1, 0], scale=2.0)
    assert chosen.tolist() == [[3, 2], [0, 1], [-1, -1]]
    assert np.allclose(w, [[0.7, 0.5], [0.5, 0.5], [0, 0]])
    assert offsets.tolist() == [0, 1, 2, 3, 4] and pairs.tolist() == [2, 3, 1, 0]


def test_the_oracle_of_the_experts():
    x, w1 = np.array([[1.0, 2.0]]), np.array([[[1.0, 0.0], [0.0, 1.0], [3.0, 0.0], [0.0, -1.0]]])
    w2 = np.array([[[1.0, 1.0], [2.0, 0.0]]])
    # gates 1, 2 (relu), ups 3, -2: h = 3, -4; down: -1, 6; weight 0.5; an expert elsewhere adds nothing
    y, _ = ffn.experts(x, w1, w2, np.array([[5, 4]]), np.array([[0.25, 0.5]]), 4, 1, 0.0, residual=np.array([[10.0, 20.0]]))
    assert y.tolist() == [[9.5, 23.0]]
