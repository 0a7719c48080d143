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


def w4_args(**kw):
    d = dict(M=4, K=512, N=256, dt=nmm.NMM_BF16, format=nmm.NMM_W4_INT, group=128, x=ALIGNED, ldx=512, Wq=ALIGNED, ldwq=256,
             scales=ALIGNED, lds=4, zeros=ALIGNED, ldz=4, y=ALIGNED, ldy=256, workspace=None, bytes=0, stream=None)
    d.update(kw)
    return tuple(d.values())


MX = dict(format=nmm.NMM_W4_MX, group=32, zeros=None, lds=16)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=7), nmm.NMM_ERR_DTYPE), (dict(format=0), nmm.NMM_ERR_DTYPE), (dict(format=3), nmm.NMM_ERR_DTYPE),
    (dict(M=-1), nmm.NMM_ERR_SHAPE), (dict(K=-1), nmm.NMM_ERR_SHAPE), (dict(N=-1), nmm.NMM_ERR_SHAPE),
    (dict(M=1 << 31), nmm.NMM_ERR_SHAPE), (dict(K=1 << 31), nmm.NMM_ERR_SHAPE), (dict(N=1 << 31), nmm.NMM_ERR_SHAPE),
    (dict(group=16), nmm.NMM_ERR_SHAPE), (dict(group=96), nmm.NMM_ERR_SHAPE), (dict(group=0), nmm.NMM_ERR_SHAPE),
    (dict(group=-32), nmm.NMM_ERR_SHAPE), (dict(MX, group=64), nmm.NMM_ERR_SHAPE), (dict(MX, zeros=ALIGNED), nmm.NMM_ERR_ARG),
    (dict(ldx=504), nmm.NMM_ERR_SHAPE), (dict(ldwq=240), nmm.NMM_ERR_SHAPE), (dict(lds=3), nmm.NMM_ERR_SHAPE),
    (dict(ldz=3), nmm.NMM_ERR_SHAPE), (dict(ldy=255), nmm.NMM_ERR_SHAPE), (dict(ldx=1 << 31), nmm.NMM_ERR_SHAPE),
    (dict(ldx=514), nmm.NMM_ERR_ALIGN), (dict(ldwq=264), nmm.NMM_ERR_ALIGN), (dict(x=ALIGNED + 8), nmm.NMM_ERR_ALIGN),
    (dict(Wq=ALIGNED + 8), nmm.NMM_ERR_ALIGN), (dict(scales=ALIGNED + 1), nmm.NMM_ERR_ALIGN),
    (dict(y=ALIGNED + 2), nmm.NMM_ERR_ALIGN), (dict(x=None), nmm.NMM_ERR_NULL), (dict(Wq=None), nmm.NMM_ERR_NULL),
    (dict(scales=None), nmm.NMM_ERR_NULL), (dict(y=None), nmm.NMM_ERR_NULL),
    (dict(N=1 << 23, ldy=1 << 23), nmm.NMM_ERR_SHAPE),                       # a weight of 2^31 bytes
    (dict(M=32, ldx=1 << 26), nmm.NMM_ERR_SHAPE),                            # 32 rows of x past 2^31 bytes
    (dict(K=16384, ldx=16384, ldwq=8192, lds=128, ldz=128), nmm.NMM_ERR_WORKSPACE),
    (dict(K=16384, ldx=16384, ldwq=8192, lds=128, ldz=128, workspace=ALIGNED, bytes=65536), nmm.NMM_ERR_WORKSPACE),
])
def test_gemv_w4_refuses(kw, status):
    assert L.nmm_gemv_w4(*w4_args(**kw)) == status


def test_gemv_w4_empty_and_workspace():
    assert L.nmm_gemv_w4(*w4_args(M=0, y=None)) == nmm.NMM_OK
    assert L.nmm_gemv_w4(*w4_args(N=0, y=None)) == nmm.NMM_OK
    size = L.nmm_gemv_w4_workspace_size
    for bad in ((-1, 512, 256, 128), (4, -1, 256, 128), (4, 512, -1, 128), (4, 512, 256, 96), (4, 512, 256, 0), (4, 512, 256, 16),
                (0, 512, 256, 128), (4, 0, 256, 128), (1 << 31, 512, 256, 128)):
        assert size(*bad) == 0
    tickets = 65536
    for M in (1, 2, 4, 5, 8, 9, 16, 17, 33, 100, 20000):
        for K in (32, 256, 257, 1536, 4099, 7168, 16384, 65536):
            for N in (1, 63, 512, 2112, 7168, 24576):
                for group in (32, 64, 128, 1024):
                    ws = size(M, K, N, group)
                    rows = 1 if M == 1 else 2 if M == 2 else 4 if M <= 4 else 8 if M <= 8 else 16 if M <= 16 else 32
                    if K <= 256:
                        assert ws == 0, (M, K, N, group)
                    if ws:      # whole partial tiles of at least two slices, no more of them than slots of K
                        assert (ws - tickets) % (rows * 64) == 0, (M, K, N, group)
                        assert ws - tickets >= 2 * rows * N * 4
                        assert ws - tickets <= -(-K // 256) * -(-M // rows) * rows * (N + 127) * 4


def batch_of(cache=None, **kw):
    a = fill(nmm.nmm_latent_attn_batch(), dict(
        batch=4, tokens=1, heads=16, q=ALIGNED, stride_qb=16 * 576, stride_qt=0, ldq=576, page_size=64, prefix_pages=ALIGNED,
        prefix_len=128, pages=ALIGNED, ld_pages=8, lens=ALIGNED, max_len=512, scale=0.04, out=ALIGNED, stride_ob=16 * 512,
        stride_ot=0, ldo=512), kw)
    a.cache = cache_of(**(cache or {}))
    return a


@pytest.mark.parametrize("cache,status", BAD_CACHE)
def test_batched_attention_refuses_a_bad_cache(cache, status):
    assert L.nmm_latent_attention_batch(ctypes.byref(batch_of(cache)), None, 0, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), nmm.NMM_ERR_SHAPE), (dict(tokens=-1), nmm.NMM_ERR_SHAPE), (dict(heads=-1), nmm.NMM_ERR_SHAPE),
    (dict(batch=1 << 20, heads=1), nmm.NMM_ERR_SHAPE), (dict(batch=1 << 14, heads=1 << 10), nmm.NMM_ERR_SHAPE),
    (dict(batch=1 << 62, tokens=4, heads=1), nmm.NMM_ERR_SHAPE),
    (dict(prefix_len=-1), nmm.NMM_ERR_SHAPE), (dict(max_len=-1), nmm.NMM_ERR_SHAPE), (dict(max_len=1 << 30), nmm.NMM_ERR_SHAPE),
    (dict(prefix_len=1 << 30), nmm.NMM_ERR_SHAPE), (dict(page_size=0), nmm.NMM_ERR_SHAPE), (dict(page_size=48), nmm.NMM_ERR_SHAPE),
    (dict(page_size=1 << 17), nmm.NMM_ERR_SHAPE), (dict(page_size=-64), nmm.NMM_ERR_SHAPE),
    (dict(ld_pages=7), nmm.NMM_ERR_SHAPE), (dict(ldq=568), nmm.NMM_ERR_SHAPE), (dict(ldo=508), nmm.NMM_ERR_SHAPE),
    (dict(stride_qb=-8), nmm.NMM_ERR_SHAPE), (dict(stride_ot=-4), nmm.NMM_ERR_SHAPE),
    (dict(ldq=580), nmm.NMM_ERR_ALIGN), (dict(stride_qb=9220), nmm.NMM_ERR_ALIGN), (dict(stride_qt=4), nmm.NMM_ERR_ALIGN),
    (dict(ldo=514), nmm.NMM_ERR_ALIGN), (dict(stride_ob=8194), nmm.NMM_ERR_ALIGN), (dict(stride_ot=2), nmm.NMM_ERR_ALIGN),
    (dict(q=ALIGNED + 8), nmm.NMM_ERR_ALIGN), (dict(out=ALIGNED + 4), nmm.NMM_ERR_ALIGN),
    (dict(pages=ALIGNED + 2), nmm.NMM_ERR_ALIGN), (dict(lens=ALIGNED + 2), nmm.NMM_ERR_ALIGN),
    (dict(prefix_pages=ALIGNED + 2), nmm.NMM_ERR_ALIGN),
    (dict(q=None), nmm.NMM_ERR_NULL), (dict(out=None), nmm.NMM_ERR_NULL), (dict(pages=None), nmm.NMM_ERR_NULL),
    (dict(lens=None), nmm.NMM_ERR_NULL), (dict(prefix_pages=None), nmm.NMM_ERR_NULL),
    (dict(scale=float("nan")), nmm.NMM_ERR_ARG), (dict(scale=float("inf")), nmm.NMM_ERR_ARG),
    (dict(), nmm.NMM_ERR_WORKSPACE),
])
def test_batched_attention_refuses(kw, status):
    assert L.nmm_latent_attention_batch(ctypes.byref(batch_of(**kw)), None, 0, None) == status


def test_batched_attention_empty_and_workspace():
    for kw in (dict(batch=0), dict(tokens=0), dict(heads=0, q=None, out=None)):
        assert L.nmm_latent_attention_batch(ctypes.byref(batch_of(**kw)), None, 0, None) == nmm.NMM_OK
    assert L.nmm_latent_attention_batch(None, None, 0, None) == nmm.NMM_ERR_NULL
    size = lambda **kw: L.nmm_latent_attention_batch_workspace_size(ctypes.byref(batch_of(**kw)))
    assert L.nmm_latent_attention_batch_workspace_size(None) == 0
    assert size(batch=-1) == 0 and size(page_size=48) == 0 and size(cache=dict(format=0)) == 0
    # one span of one kind of positions needs no partial results, nor does nothing at all
    assert size(prefix_len=0, max_len=64) == 0 and size(max_len=0, prefix_len=64) == 0 and size(prefix_len=0, max_len=0) == 0
    per_slot = lambda rows: rows * (512 + 2) * 4
    for batch, heads, prefix, own in ((1, 1, 1, 1), (4, 16, 128, 512), (1, 128, 0, 100000), (64, 16, 0, 4097), (3, 7, 100000, 1),
                                      (1, 1, (1 << 30) - 1, (1 << 30) - 1)):
        ws = size(batch=batch, heads=heads, prefix_len=prefix, max_len=own)
        if prefix and own:
            assert ws
        if ws:
            slots, rest = divmod(ws - 65536, per_slot(batch * heads))
            assert rest == 0 and 2 <= slots <= 64, (batch, heads, prefix, own)


STRUCTS = {"nmm_latent_cache": ["data", "rows", "ld", "kv_lora", "rope", "format"],
           "nmm_cache_entries": ["tokens", "src", "src_type", "ld_src", "slots", "gamma", "eps", "positions", "rope_theta"],
           "nmm_latent_attn_batch": ["batch", "tokens", "heads", "q", "stride_qb", "stride_qt", "ldq", "cache", "page_size",
                                     "prefix_pages", "prefix_len", "pages", "ld_pages", "lens", "max_len", "scale", "out",
                                     "stride_ob", "stride_ot", "ldo"]}


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


def test_packed_arguments_match_the_structs():
    c = cache_of(data=1 << 40, rows=7, ld=672, rope=32, kv_lora=256, format=nmm.NMM_CACHE_BF16)
    pool = (1 << 40, 7, 672, 256, 32, nmm.NMM_CACHE_BF16)
    assert nmm._CACHE.pack(*pool) == bytes(c)
    e = entries_of(tokens=3, src=1 << 41, src_type=nmm.NMM_SRC_BF16, ld_src=584, slots=1 << 42, gamma=None, eps=0.5, positions=8,
                   rope_theta=2.0)
    assert nmm._ENTRIES.pack(3, 1 << 41, nmm.NMM_SRC_BF16, 584, 1 << 42, 0, 0.5, 8, 2.0) == bytes(e)
    a = batch_of(dict(data=1 << 40, rows=7, ld=672, rope=32, kv_lora=256, format=nmm.NMM_CACHE_BF16), batch=2, tokens=3, heads=5,
                 q=1 << 43, stride_qb=11, stride_qt=12, ldq=13, page_size=16, prefix_pages=1 << 44, prefix_len=17, pages=1 << 45,
                 ld_pages=18, lens=1 << 46, max_len=19, scale=0.25, out=1 << 47, stride_ob=20, stride_ot=21, ldo=22)
    assert nmm._ATTN_BATCH.pack(2, 3, 5, 1 << 43, 11, 12, 13, *pool, 16, 1 << 44, 17, 1 << 45, 18, 1 << 46, 19, 0.25, 1 << 47, 20,
                                21, 22) == bytes(a)


@pytest.mark.parametrize("kw,status", [
    (dict(stride_ob=508), nmm.NMM_ERR_SHAPE), (dict(stride_ob=0), nmm.NMM_ERR_SHAPE),
    (dict(tokens=2, stride_ot=508, stride_ob=32 * 512), nmm.NMM_ERR_SHAPE), (dict(tokens=2, stride_ot=0), nmm.NMM_ERR_SHAPE),
    # an axis of one has no rows to lie over each other, and q may be one row for all
    (dict(batch=1, stride_ob=0), nmm.NMM_ERR_WORKSPACE), (dict(stride_ot=0), nmm.NMM_ERR_WORKSPACE),
    (dict(heads=8, tokens=2, stride_ot=512, ldo=1024), nmm.NMM_ERR_WORKSPACE),
    (dict(stride_qb=0), nmm.NMM_ERR_WORKSPACE), (dict(tokens=2, stride_ot=16 * 512, stride_ob=32 * 512), nmm.NMM_ERR_WORKSPACE),
])
def test_batched_attention_refuses_outputs_over_each_other(kw, status):
    assert L.nmm_latent_attention_batch(ctypes.byref(batch_of(**kw)), None, 0, None) == status
