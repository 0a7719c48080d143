"""The batched decode's entry points without a GPU: every invalid argument is refused before the device is touched."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
nmm = pytest.importorskip("paper_2609_16009_amd")
if not os.path.exists(nmm.LIB_PATH):
    pytest.skip("libnmm.so not built", allow_module_level=True)

L = nmm.lib()
ALIGNED = 1 << 20          # a fake, 256-byte aligned "device address"; never dereferenced here


def fill(struct, defaults, kw):
    for k, v in defaults.items():
        setattr(struct, k, kw[k] if k in kw else v)
    return struct


def cache_of(**kw):
    return fill(nmm.nmm_latent_cache(), dict(data=ALIGNED, rows=1000, ld=656, kv_lora=512, rope=64,
                                             format=nmm.NMM_CACHE_E4M3), kw)


def entries_of(**kw):
    return fill(nmm.nmm_cache_entries(), dict(tokens=4, src=ALIGNED, src_type=nmm.NMM_SRC_F32, ld_src=576, slots=ALIGNED,
                                              gamma=ALIGNED, eps=1e-6, positions=ALIGNED, rope_theta=1e4), kw)


BAD_CACHE = [
    (dict(format=0), nmm.NMM_ERR_DTYPE), (dict(format=3), nmm.NMM_ERR_DTYPE),
    (dict(kv_lora=0), nmm.NMM_ERR_SHAPE), (dict(kv_lora=520), nmm.NMM_ERR_SHAPE), (dict(kv_lora=544), nmm.NMM_ERR_SHAPE),
    (dict(kv_lora=-32), nmm.NMM_ERR_SHAPE), (dict(rope=4), nmm.NMM_ERR_SHAPE), (dict(rope=72), nmm.NMM_ERR_SHAPE),
    (dict(rope=-8), nmm.NMM_ERR_SHAPE), (dict(rows=-1), nmm.NMM_ERR_SHAPE), (dict(rows=1 << 31), nmm.NMM_ERR_SHAPE),
    (dict(ld=640), nmm.NMM_ERR_SHAPE), (dict(ld=1 << 31), nmm.NMM_ERR_SHAPE),
    (dict(ld=1136, format=nmm.NMM_CACHE_BF16), nmm.NMM_ERR_SHAPE), (dict(ld=660), nmm.NMM_ERR_ALIGN),
    (dict(data=ALIGNED + 8), nmm.NMM_ERR_ALIGN), (dict(data=None), nmm.NMM_ERR_NULL),
]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_every_call_refuses_a_bad_cache(kw, status):
    c, e = cache_of(**kw), entries_of()
    assert L.nmm_latent_cache_write(ctypes.byref(c), ctypes.byref(e), None) == status
    assert L.nmm_latent_cache_read(ctypes.byref(c), 4, ALIGNED, ALIGNED, 576, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(src_type=2), nmm.NMM_ERR_DTYPE), (dict(tokens=-1), nmm.NMM_ERR_SHAPE), (dict(tokens=1 << 31), nmm.NMM_ERR_SHAPE),
    (dict(tokens=1 << 30), nmm.NMM_ERR_SHAPE), (dict(ld_src=572), nmm.NMM_ERR_SHAPE), (dict(ld_src=1 << 31), nmm.NMM_ERR_SHAPE),
    (dict(ld_src=578), nmm.NMM_ERR_ALIGN), (dict(ld_src=580, src_type=nmm.NMM_SRC_BF16), nmm.NMM_ERR_ALIGN),
    (dict(src=ALIGNED + 4), nmm.NMM_ERR_ALIGN), (dict(gamma=ALIGNED + 2), nmm.NMM_ERR_ALIGN),
    (dict(slots=ALIGNED + 4), nmm.NMM_ERR_ALIGN), (dict(positions=ALIGNED + 4), nmm.NMM_ERR_ALIGN),
    (dict(src=None), nmm.NMM_ERR_NULL), (dict(slots=None), nmm.NMM_ERR_NULL),
    (dict(eps=-1.0), nmm.NMM_ERR_ARG), (dict(eps=float("nan")), nmm.NMM_ERR_ARG),
    (dict(rope_theta=0.0), nmm.NMM_ERR_ARG), (dict(rope_theta=float("inf")), nmm.NMM_ERR_ARG),
])
def test_cache_write_refuses(kw, status):
    c, e = cache_of(), entries_of(**kw)
    assert L.nmm_latent_cache_write(ctypes.byref(c), ctypes.byref(e), None) == status


@pytest.mark.parametrize("tokens,slots,out,ldo,status", [
    (-1, ALIGNED, ALIGNED, 576, nmm.NMM_ERR_SHAPE), (1 << 31, ALIGNED, ALIGNED, 576, nmm.NMM_ERR_SHAPE),
    (1 << 30, ALIGNED, ALIGNED, 576, nmm.NMM_ERR_SHAPE), (4, ALIGNED, ALIGNED, 568, nmm.NMM_ERR_SHAPE),
    (4, None, ALIGNED, 576, nmm.NMM_ERR_NULL), (4, ALIGNED, None, 576, nmm.NMM_ERR_NULL),
    (4, ALIGNED + 4, ALIGNED, 576, nmm.NMM_ERR_ALIGN), (4, ALIGNED, ALIGNED + 2, 576, nmm.NMM_ERR_ALIGN),
    (4, ALIGNED, ALIGNED, 580, nmm.NMM_ERR_ALIGN),
])
def test_cache_read_refuses(tokens, slots, out, ldo, status):
    assert L.nmm_latent_cache_read(ctypes.byref(cache_of()), tokens, slots, out, ldo, None) == status


def test_empty_cache_calls_are_noops():
    c, none = cache_of(), cache_of(rows=0, data=None)
    assert L.nmm_latent_cache_write(ctypes.byref(c), ctypes.byref(entries_of(tokens=0, src=None)), None) == nmm.NMM_OK
    assert L.nmm_latent_cache_write(ctypes.byref(none), ctypes.byref(entries_of()), None) == nmm.NMM_OK
    assert L.nmm_latent_cache_read(ctypes.byref(c), 0, None, None, 576, None) == nmm.NMM_OK
    assert L.nmm_latent_cache_read(ctypes.byref(none), 4, ALIGNED, ALIGNED, 576, None) == nmm.NMM_OK
    assert L.nmm_latent_cache_write(None, ctypes.byref(entries_of()), None) == nmm.NMM_ERR_NULL
    assert L.nmm_latent_cache_write(ctypes.byref(c), None, None) == nmm.NMM_ERR_NULL
    assert L.nmm_latent_cache_read(None, 4, ALIGNED, ALIGNED, 576, None) == nmm.NMM_ERR_NULL


def test_row_bytes():
    assert nmm.nmm_latent_cache_row_bytes(512, 64) == 656
    assert nmm.nmm_latent_cache_row_bytes(512, 64, nmm.NMM_CACHE_BF16) == 1152
    assert nmm.nmm_latent_cache_row_bytes(32, 0) == 48
    for bad in ((513, 64, 2), (0, 0, 1), (544, 0, 2), (64, 7, 2), (64, 8, 5)):
        assert nmm.nmm_latent_cache_row_bytes(*bad) == 0


STRUCTS = {"nmm_latent_cache": ["data", "rows", "ld", "kv_lora", "rope", "format"],
           "nmm_cache_entries": ["tokens", "src", "src_type", "ld_src", "slots", "gamma", "eps", "positions", "rope_theta"]}


def test_struct_layouts_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "nmm.h"', "int main(void) {"]
    for st, fields in STRUCTS.items():
        lines.append(f'  printf("{st} sizeof %zu\\n", sizeof({st}));')
        lines += [f'  printf("{st} {f} %zu\\n", offsetof({st}, {f}));' for f in fields]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = {tuple(l.split()[:2]): int(l.split()[2]) for l in subprocess.run([str(exe)], capture_output=True, text=True,
                                                                           check=True).stdout.split("\n") if l}
    for st, fields in STRUCTS.items():
        cls = getattr(nmm, st)
        assert got[(st, "sizeof")] == ctypes.sizeof(cls), st
        for f in fields:
            assert got[(st, f)] == getattr(cls, f).offset, (st, f)
