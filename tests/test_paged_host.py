"""Host-side checks of the paged cache's C ABI (no GPU needed): every refusal comes before
anything is launched, the descriptor is laid out as the C compiler does, and the host code is clean
under AddressSanitizer and UndefinedBehaviorSanitizer."""
import ctypes
import os
import subprocess

import pytest

import paper_2505_22913_amd as mf
from tests.test_sanitizers import CLANG, CSRC, ENV, HIPCC, ROOT, SAN, _run, needs_toolchain

HEADER = os.path.join(ROOT, "include")
BUFFERS = dict(k=0x100000, v=0x200000, table=0x300000, state=0x400000, free_pages=0x500000)
SHAPE = dict(B=3, H=8, d=128, page_tokens=64, n_pages=100, max_pages=40, type=mf.FP16)
STRIDES = dict(page_stride=8 * 64 * 128, head_stride=64 * 128, token_stride=128)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mf.LIB_PATH):
        from paper_2505_22913_amd import build_lib
        build_lib.build()
    return mf.lib()


def init(**kw):
    a = {**BUFFERS, **SHAPE, **STRIDES, **kw}
    p = mf.pages_t()
    return p, mf.lib().mustafar_paged_init(ctypes.byref(p), *a.values())


def test_struct_layout_matches_the_c_compiler(tmp_path):
    names = [n for n, _ in mf.pages_t._fields_]
    prog = tmp_path / "layout.c"
    prog.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mustafar.h"\nint main(void){printf("%zu", '
                    "sizeof(mustafar_pages_t));" + "".join(f'printf(" %zu", offsetof(mustafar_pages_t, {n}));' for n in names)
                    + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", f"-I{HEADER}", "-o", str(exe), str(prog)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(mf.pages_t)] + [getattr(mf.pages_t, n).offset for n in names]


def test_init_checks_the_descriptor(lib):
    p, st = init()
    assert st == mf.OK and (p.B, p.H, p.n_pages, p.token_stride) == (3, 8, 100, 128)
    for ok in (dict(d=64), dict(d=256, page_stride=8 * 64 * 256, head_stride=64 * 256, token_stride=256), dict(page_tokens=16),
               dict(type=mf.BF16), dict(head_stride=128, token_stride=8 * 128), dict(B=4096), dict(n_pages=1, page_stride=128),
               dict(page_stride=1 << 40)):
        assert init(**ok)[1] == mf.OK, ok
    for bad in (dict(k=0), dict(k=0x100008), dict(v=0x200002), dict(table=0), dict(state=0x400002), dict(free_pages=0x500001),
                dict(B=0), dict(B=4097), dict(H=0), dict(d=96), dict(d=0), dict(d=256), dict(page_tokens=8),
                dict(page_tokens=48), dict(page_tokens=2048), dict(n_pages=0), dict(n_pages=1 << 25), dict(max_pages=0),
                dict(max_pages=(1 << 19) + 1), dict(type=2), dict(type=-1), dict(page_stride=8 * 64 * 128 - 8),
                dict(token_stride=120), dict(head_stride=64 * 128 - 8), dict(head_stride=64 * 128 + 4),
                dict(token_stride=132), dict(head_stride=120, token_stride=1024), dict(page_stride=(1 << 40) + 8),
                dict(head_stride=1 << 28, page_stride=1 << 40), dict(head_stride=-8192)):
        assert init(**bad)[1] == mf.EINVAL, bad
    assert lib.mustafar_paged_init(None, *{**BUFFERS, **SHAPE, **STRIDES}.values()) == mf.EINVAL


def broken():
    """A descriptor that was spoilt after its init."""
    p, _ = init()
    p.page_tokens = 17
    return p


def test_plan_refuses(lib):
    p, _ = init()
    args = dict(keep=None, new_len=0x10, state_out=0x400000, cu=0x20, slots=0x30, n_slots=5, status=0x40)
    for bad in (dict(keep=0x12), dict(new_len=0), dict(new_len=0x11), dict(state_out=0), dict(cu=0), dict(slots=0),
                dict(slots=0x31), dict(n_slots=-1), dict(n_slots=(1 << 19) + 1), dict(status=0),
                dict(state_out=0x400004), dict(state_out=0x400000 - 16)):
        assert lib.mustafar_paged_plan(ctypes.byref(p), *{**args, **bad}.values(), None) == mf.EINVAL, bad
    assert lib.mustafar_paged_plan(ctypes.byref(broken()), *args.values(), None) == mf.EINVAL
    assert lib.mustafar_paged_plan(None, *args.values(), None) == mf.EINVAL


def test_write_and_gather_refuse(lib):
    p, _ = init()
    args = dict(k=0x10, ks=1024, v=0x20, vs=1024, slots=0x30, n=4)
    for bad in (dict(k=0), dict(k=0x18), dict(v=0x24), dict(ks=1016), dict(ks=1028), dict(vs=-1024), dict(vs=1 << 32),
                dict(slots=0), dict(slots=0x32), dict(n=-1)):
        assert lib.mustafar_paged_write(ctypes.byref(p), *{**args, **bad}.values(), None) == mf.EINVAL, bad
    assert lib.mustafar_paged_write(ctypes.byref(broken()), *args.values(), None) == mf.EINVAL
    assert lib.mustafar_paged_write(ctypes.byref(p), None, 0, None, 0, None, 0, None) == mf.OK     # nothing to do
    args = dict(first=None, x_k=0x10, x_v=0x20, n=4)
    for bad in (dict(first=0x11), dict(x_k=0), dict(x_k=0x18), dict(x_v=0x22), dict(n=-1)):
        assert lib.mustafar_paged_gather(ctypes.byref(p), *{**args, **bad}.values(), None) == mf.EINVAL, bad
    assert lib.mustafar_paged_gather(ctypes.byref(broken()), *args.values(), None) == mf.EINVAL
    assert lib.mustafar_paged_gather(ctypes.byref(p), None, None, None, 0, None) == mf.OK


def attn(p, **kw):
    a = dict(q=0x10, qs=32 * 128, n_q=5, Hq=32, p=ctypes.byref(p), cu=0x20, window=0, sinks=0, scale=0.0, out=0x30,
             os=32 * 128, max_q=5, max_tokens=5000, n_splits=0, ws=0x1000, ws_bytes=1 << 40, stream=None)
    return mf.lib().mustafar_paged_attn(*{**a, **kw}.values())


def test_attention_refuses(lib):
    p, _ = init()
    for bad in (dict(q=0), dict(q=0x18), dict(qs=32 * 128 - 8), dict(qs=32 * 128 + 4), dict(qs=1 << 32), dict(n_q=-1),
                dict(Hq=0), dict(Hq=33), dict(cu=0), dict(cu=0x22), dict(window=-1), dict(sinks=-1), dict(out=0),
                dict(out=0x38), dict(os=128), dict(max_q=-1), dict(max_tokens=-1), dict(n_splits=(1 << 16) + 1),
                dict(n_q=0x7fffffff)):
        assert attn(p, **bad) == mf.EINVAL, bad
    assert attn(p, Hq=8 * 65, qs=8 * 65 * 128, os=8 * 65 * 128) == mf.EUNSUPPORTED
    assert attn(broken()) == mf.EINVAL
    assert attn(p, n_q=0, q=0, out=0, cu=0) == mf.OK      # nothing to do


@needs_toolchain
def test_paged_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                "-Xarch_host", "-fno-sanitize-recover=all"]
    common = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fno-strict-aliasing", f"-I{HEADER}", f"-I{CSRC}"]
    objs = []
    for src in (os.path.join(CSRC, "paged_api.hip"), os.path.join(SAN, "paged_stubs.hip")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([HIPCC, *common, *host_san, "-c", src, "-o", objs[-1]])
    objs.append(str(tmp_path / "harness.o"))
    _run([CLANG, "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", f"-I{HEADER}", "-c",
          os.path.join(SAN, "paged_harness.c"), "-o", objs[-1]])
    exe = str(tmp_path / "paged_harness")
    _run([HIPCC, "-fsanitize=address,undefined", "-fno-gpu-sanitize", *objs, "-o", exe])
    assert "paged harness ok" in _run([exe], env=ENV)


def test_a_workspace_does_for_every_shorter_length(lib):
    """A call's ranges follow what its rows see, its workspace max_tokens: more of these never need less."""
    for kw in (dict(), dict(B=1), dict(B=64), dict(d=64, page_stride=8 * 64 * 64, head_stride=64 * 64, token_stride=64)):
        p, st = init(**kw)
        assert st == mf.OK
        for Hq, n_q, max_q in ((8, 64, 1), (32, 3, 1), (32, 64, 2), (8, 300, 100), (32, 512, 512), (64, 6000, 2000), (32, 200, 60)):
            last = 0
            for tokens in list(range(0, 3000, 97)) + [4096, 10000, 32768, 100000, 1 << 22, 2 ** 31 - 1]:
                need = lib.mustafar_paged_attn_workspace_bytes(ctypes.byref(p), Hq, n_q, max_q, tokens, 0)
                assert need >= last, (kw, Hq, n_q, max_q, tokens)
                last = need


def pages(**kw):
    d, H = kw.get("d", 128), kw.get("H", 8)
    p, st = init(**{"d": d, "H": H, "page_stride": H * 64 * d, "head_stride": 64 * d, "token_stride": d, "n_pages": 1 << 20,
                    "max_pages": 1 << 15, **kw})
    assert st == mf.OK
    return p


def need(p, Hq, n_q, max_q, max_tokens, n_splits=0):
    return mf.lib().mustafar_paged_attn_workspace_bytes(ctypes.byref(p), Hq, n_q, max_q, max_tokens, n_splits)


@pytest.mark.parametrize("B,H,Hq,n_q,max_q,tokens", [
    (2, 8, 32, 8193, 8192, 32768), (2, 1, 8, 8193, 8192, 131072), (2, 8, 32, 513, 512, 16384), (2, 8, 32, 16385, 16384, 32768),
    (4, 32, 32, 16384, 16384, 4096), (2, 1, 1, 100001, 100000, 200000), (64, 8, 32, 9000, 8192, 131072)])
def test_a_long_chunk_beside_single_tokens_needs_a_small_workspace(lib, B, H, Hq, n_q, max_q, tokens):
    """Single tokens' ranges are paid for by the rows that single tokens can have, not by the chunk's."""
    for d in (64, 128, 256):
        assert need(pages(B=B, H=H, d=d), Hq, n_q, max_q, tokens) <= 60 << 20, d


def test_no_call_needs_more_than_the_launches_rows(lib):
    """With the split that calls take by themselves: at most 16 * 2048 + 256 * 256 rows, as the header says."""
    sizes = [1, 2, 3, 7, 16, 17, 63, 64, 65, 200, 512, 1000, 4096, 5000, 30000, 200000]
    for d, rows in ((64, 98304), (128, 98304), (256, 98304)):
        most = 0
        for B in (1, 2, 3, 17, 64, 500, 4096):
            for H, G in ((1, 1), (1, 64), (2, 3), (8, 4), (8, 16), (8, 17), (32, 1)):
                p = pages(B=B, H=H, d=d)
                for n_q in sizes:
                    for max_q in [0] + sizes:
                        most = max(most, need(p, H * G, n_q, max_q, 2 ** 21))
        assert 1 << 24 <= most <= rows * (d + 2) * 4


@needs_toolchain
def test_launches_of_too_many_threads_are_refused(tmp_path):
    """Against stubs of the launchers, so that what is accepted launches nothing."""
    objs = []
    for src in (os.path.join(CSRC, "paged_api.hip"), os.path.join(SAN, "paged_stubs.hip")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", f"-I{HEADER}", f"-I{CSRC}", "-c", src, "-o", objs[-1]])
    objs.append(str(tmp_path / "limits.o"))
    _run([CLANG, "-O1", f"-I{HEADER}", "-c", os.path.join(SAN, "paged_limits.c"), "-o", objs[-1]])
    exe = str(tmp_path / "paged_limits")
    _run([HIPCC, *objs, "-o", exe])
    assert "paged limits ok" in _run([exe], env=ENV)
