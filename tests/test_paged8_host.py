"""Host-side checks of the C ABI of the 8-bit paged cache and of rotary positions (no GPU needed): every refusal comes
before anything is launched, the descriptors are laid out as the C compiler does, rates are the formulas', and the host
code is clean under AddressSanitizer and UndefinedBehaviorSanitizer."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2505_22913_amd as mf
from oracle import paged8 as oracle8
from tests.test_sanitizers import CLANG, CSRC, ENV, HIPCC, ROOT, SAN, _run, needs_toolchain

HEADER = os.path.join(ROOT, "include")
BUFFERS = dict(k=0x100000, v=0x200000, k_scale=0x600001, v_scale=0x700003, table=0x300000, state=0x400000, free_pages=0x500000)
SHAPE = dict(B=3, H=8, d=128, page_tokens=64, n_pages=100, max_pages=40, type=mf.FP16, code=mf.E4M3, block_tokens=16)
STRIDES = dict(page_stride=8 * 64 * 128, head_stride=64 * 128, token_stride=128)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mf.LIB_PATH):
        from paper_2505_22913_amd import build_lib
        build_lib.build()
    return mf.lib()


def init(**kw):
    a = {**BUFFERS, **SHAPE, **STRIDES, **kw}
    p = mf.pages8_t()
    return p, mf.lib().mustafar_paged8_init(ctypes.byref(p), *a.values())


@pytest.mark.parametrize("struct", ["pages8", "rotation"])
def test_struct_layouts_match_the_c_compiler(tmp_path, struct):
    mirror = getattr(mf, struct + "_t")
    names = [n for n, _ in mirror._fields_]
    prog = tmp_path / "layout.c"
    prog.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mustafar.h"\nint main(void){printf("%zu", '
                    f"sizeof(mustafar_{struct}_t));" + "".join(f'printf(" %zu", offsetof(mustafar_{struct}_t, {n}));' for n in names)
                    + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", f"-I{HEADER}", "-o", str(exe), str(prog)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(mirror)] + [getattr(mirror, n).offset for n in names]


def test_init_checks_the_descriptor(lib):
    p, st = init()
    assert st == mf.OK and (p.pages.B, p.pages.type, p.type, p.block_tokens) == (3, mf.E4M3, mf.FP16, 16)
    for ok in (dict(code=mf.INT8, type=mf.BF16), dict(block_tokens=32), dict(block_tokens=64), dict(page_tokens=16),
               dict(head_stride=128, token_stride=8 * 128), dict(d=64, page_stride=8 * 64 * 64, head_stride=64 * 64, token_stride=64)):
        assert init(**ok)[1] == mf.OK, ok
    for bad in (dict(k=0), dict(k=0x100008), dict(v=0x200002), dict(k_scale=0), dict(v_scale=0), dict(table=0), dict(state=0x400002),
                dict(free_pages=0), dict(B=0), dict(B=4097), dict(H=0), dict(d=96), dict(page_tokens=8), dict(n_pages=0),
                dict(n_pages=1 << 25), dict(max_pages=0), dict(type=mf.E4M3), dict(type=-1), dict(code=mf.FP16), dict(code=mf.BF16),
                dict(code=4), dict(block_tokens=0), dict(block_tokens=8), dict(block_tokens=48), dict(block_tokens=128, page_tokens=256),
                dict(block_tokens=32, page_tokens=16), dict(token_stride=136, head_stride=64 * 136, page_stride=8 * 64 * 136),
                dict(page_stride=8 * 64 * 128 + 8), dict(head_stride=64 * 128 + 8, page_stride=9 * 64 * 128),
                dict(page_stride=8 * 64 * 128 - 16), dict(page_stride=(1 << 40) + 16), dict(head_stride=-8192)):
        assert init(**bad)[1] == mf.EINVAL, bad
    assert lib.mustafar_paged8_init(None, *{**BUFFERS, **SHAPE, **STRIDES}.values()) == mf.EINVAL


def test_pages_of_codes_are_refused_by_the_dense_calls_and_taken_by_the_plan(lib):
    p, _ = init()
    pages = ctypes.byref(p.pages)
    assert lib.mustafar_paged_write(pages, 0x10, 1024, 0x20, 1024, 0x30, 4, None) == mf.EINVAL
    assert lib.mustafar_paged_gather(pages, None, 0x10, 0x20, 4, None) == mf.EINVAL
    assert lib.mustafar_paged_attn(0x10, 4096, 5, 32, pages, 0x20, 0, 0, 0.0, 0x30, 4096, 5, 5000, 0, 0x1000, 1 << 40, None) == mf.EINVAL
    assert lib.mustafar_paged_attn_workspace_bytes(pages, 32, 5, 5, 5000, 4) == 0
    assert lib.mustafar_paged_plan(pages, None, 0, 0x400000, 0x20, 0x30, 5, 0x40, None) == mf.EINVAL      # for its arguments alone
    q = mf.pages8_t.from_buffer_copy(p)
    q.pages.type = mf.FP16
    assert lib.mustafar_paged8_gather(ctypes.byref(q), None, 0x10, 0x20, 4, None) == mf.EINVAL


def broken():
    """A descriptor that was spoilt after its init."""
    p, _ = init()
    p.block_tokens = 17
    return p


def test_write_and_gather_refuse(lib):
    p, _ = init()
    args = dict(k=0x10, ks=1024, v=0x20, vs=1024, cu=0x30, n=4)
    for bad in (dict(k=0), dict(k=0x18), dict(v=0x24), dict(ks=1016), dict(ks=1028), dict(vs=-1024), dict(vs=1 << 32), dict(cu=0),
                dict(cu=0x32), dict(n=-1), dict(n=2 ** 31 - 1)):
        assert lib.mustafar_paged8_write(ctypes.byref(p), *{**args, **bad}.values(), None) == mf.EINVAL, bad
    assert lib.mustafar_paged8_write(ctypes.byref(broken()), *args.values(), None) == mf.EINVAL
    assert lib.mustafar_paged8_write(ctypes.byref(p), None, 0, None, 0, None, 0, None) == mf.OK     # nothing to do
    args = dict(first=None, x_k=0x10, x_v=0x20, n=4)
    for bad in (dict(first=0x11), dict(x_k=0), dict(x_k=0x18), dict(x_v=0x22), dict(n=-1), dict(n=2 ** 31 - 1)):
        assert lib.mustafar_paged8_gather(ctypes.byref(p), *{**args, **bad}.values(), None) == mf.EINVAL, bad
    assert lib.mustafar_paged8_gather(ctypes.byref(broken()), *args.values(), None) == mf.EINVAL
    assert lib.mustafar_paged8_gather(ctypes.byref(p), None, None, None, 0, None) == mf.OK


def attn(p, **kw):
    a = dict(q=0x10, qs=32 * 128, n_q=5, Hq=32, p=ctypes.byref(p), cu=0x20, window=0, sinks=0, scale=0.0, out=0x30,
             os=32 * 128, max_q=5, max_tokens=5000, n_splits=0, ws=0x1000, ws_bytes=1 << 40, stream=None)
    return mf.lib().mustafar_paged8_attn(*{**a, **kw}.values())


def test_attention_refuses(lib):
    p, _ = init()
    for bad in (dict(q=0), dict(q=0x18), dict(qs=32 * 128 - 8), dict(qs=32 * 128 + 4), dict(qs=1 << 32), dict(n_q=-1),
                dict(Hq=0), dict(Hq=33), dict(cu=0), dict(cu=0x22), dict(window=-1), dict(sinks=-1), dict(out=0),
                dict(out=0x38), dict(os=128), dict(max_q=-1), dict(max_tokens=-1), dict(n_splits=(1 << 16) + 1),
                dict(n_q=0x7fffffff)):
        assert attn(p, **bad) == mf.EINVAL, bad
    assert attn(p, Hq=8 * 65, qs=8 * 65 * 128, os=8 * 65 * 128) == mf.EUNSUPPORTED
    assert attn(p, n_splits=4, ws_bytes=100) == mf.EWORKSPACE and attn(p, n_splits=4, ws=0x1008) == mf.EWORKSPACE
    assert attn(broken()) == mf.EINVAL
    assert attn(p, n_q=0, q=0, out=0, cu=0) == mf.OK      # nothing to do


def test_a_workspace_does_for_every_shorter_length_and_stays_in_its_bound(lib):
    for kw in (dict(), dict(B=1), dict(B=64), dict(B=4096, H=1, page_stride=64 * 128),
               dict(d=256, page_stride=8 * 64 * 256, head_stride=64 * 256, token_stride=256)):
        p, st = init(**kw)
        assert st == mf.OK
        H, d = p.pages.H, p.pages.d
        for Hq, n_q, max_q in ((8, 64, 1), (32, 3, 1), (32, 64, 2), (8, 300, 100), (32, 512, 512), (64, 6000, 2000), (32, 200, 60), (8, 1, 1),
                               (8, 8193, 8192), (64, 4097, 4096)):
            last = 0
            for tokens in list(range(0, 3000, 97)) + [4096, 10000, 32768, 100000, 1 << 22, 2 ** 31 - 1]:
                need = lib.mustafar_paged8_attn_workspace_bytes(ctypes.byref(p), Hq, n_q, max_q, tokens, 0)
                assert last <= need <= 393216 * (d + 2), (kw, Hq, n_q, max_q, tokens)
                last = need


# ---- rotary positions ----------------------------------------------------------------------------
@pytest.mark.parametrize("rot", [2, 4, 20, 64, 128, 512])
@pytest.mark.parametrize("scaling,kw", [("plain", {}), ("plain", dict(factor=-3.0)), ("linear", dict(factor=8.0)), ("base", dict(factor=4.0)),
                                        ("turns", dict(factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=4.0)),
                                        ("turns", dict(factor=32.0, original_len=4096.0, low_turns=1.0, high_turns=32.0))])
def test_rates_are_the_formulas(lib, rot, scaling, kw):
    if scaling == "base" and rot == 2:
        with pytest.raises(mf.MustafarError):
            mf.mustafar_rope_rates(rot, 10000.0, scaling, **kw)
        return
    got = mf.mustafar_rope_rates(rot, 10000.0, scaling, **kw)
    want = oracle8.rates(rot, 10000.0, scaling, kw.get("factor", 1.0), kw.get("original_len", 0.0), kw.get("low_turns", 1), kw.get("high_turns", 32))
    assert len(got) == rot // 2 and all(abs(a - b) <= 1e-14 * b for a, b in zip(got, want))
    if scaling == "base":       # the first stays, the last is divided
        assert got[0] == 1 and abs(got[-1] * kw["factor"] / 10000.0 ** (-(rot - 2) / rot) - 1) < 1e-12


@pytest.mark.parametrize("rot,base,factor", [(8, 1e300, 1e10), (4, 1e160, 1e100), (64, 1e307, 16.0), (128, 1e-300, 1e-7), (6, 1e-200, 1e-100),
                                             (64, 1e300, 1e-280)])
def test_an_enlarged_base_beyond_doubles_range_has_its_rates(lib, rot, base, factor):
    """base * factor^(rot / (rot - 2)) may leave fp64's range where its powers do not (the last pair's exponent is under 1): their logarithms,
    off by 2^-52 of themselves, which are under 1500, and as little from the powers' own roundings."""
    got = mf.mustafar_rope_rates(rot, base, "base", factor=factor)
    for i, r in enumerate(got):
        want = -2 * i / rot * (math.log(base) + rot / (rot - 2) * math.log(factor))
        assert r > 0 and abs(math.log(r) - want) <= 8 * 1500 * 2.0 ** -52, (i, r, want)
    assert got[0] == 1 and all(a > b if base > 1 else a < b for a, b in zip(got, got[1:]))


def test_rates_refuse(lib):
    out = (ctypes.c_double * 256)(*[7.0] * 256)
    call = lambda rot=64, base=1e4, scaling=0, factor=2.0, L=4096.0, low=1.0, high=4.0, r=out: lib.mustafar_rope_rates(  # noqa: E731
        r, rot, base, scaling, factor, L, low, high)
    nan, inf = math.nan, math.inf
    for bad in (dict(rot=0), dict(rot=1), dict(rot=63), dict(rot=514), dict(rot=-2), dict(base=0.0), dict(base=-1.0), dict(base=nan),
                dict(base=inf), dict(scaling=-1), dict(scaling=4), dict(scaling=1, factor=0.0), dict(scaling=1, factor=nan),
                dict(scaling=2, factor=-2.0), dict(scaling=2, rot=2), dict(scaling=3, L=0.0), dict(scaling=3, L=nan), dict(scaling=3, low=4.0),
                dict(scaling=3, high=inf), dict(scaling=3, low=nan), dict(base=1e-300, scaling=2, factor=1e-300), dict(r=None)):
        assert call(**bad) == mf.EINVAL, bad
    assert all(x == 7.0 for x in out)       # a refused call writes nothing


def rope(**kw):
    r = mf.rotation_t(kw.pop("rates", 0x8), kw.pop("rot", 64), kw.pop("layout", 0), 1.0)
    a = dict(r=ctypes.byref(r), q=0x10, qs=512, Hq=4, k=0x20, ks=256, H=2, d=128, n=5, type=mf.FP16, positions=0x30, p=None, cu=None,
             inverse=0, out_q=0x40, oqs=512, out_k=0x50, oks=256, stream=None)
    return mf.lib().mustafar_rope(*{**a, **kw}.values())


def test_rope_refuses(lib):
    p, _ = init()
    pages = ctypes.byref(p.pages)
    for bad in (dict(r=None), dict(rates=0), dict(rates=0xc), dict(rot=0), dict(rot=63), dict(rot=130), dict(layout=2), dict(layout=-1),
                dict(q=0), dict(q=0x18), dict(qs=504), dict(qs=516), dict(qs=1 << 32), dict(k=0), dict(ks=248), dict(H=0), dict(Hq=0),
                dict(Hq=-1), dict(H=1 << 17), dict(d=0), dict(d=132), dict(d=520), dict(n=-1), dict(type=2), dict(type=-1),
                dict(positions=0), dict(positions=0x32), dict(cu=0x40), dict(p=pages), dict(positions=0, p=pages), dict(positions=0, cu=0x40),
                dict(positions=0, p=pages, cu=0x42), dict(out_q=0), dict(out_q=0x48), dict(oqs=8), dict(out_k=0), dict(out_q=0x10, oqs=520),
                dict(out_k=0x20, oks=264), dict(q=0, Hq=0, k=0, H=0, out_q=0, out_k=0), dict(n=2 ** 31 - 1, Hq=1 << 16, qs=1 << 23, oqs=1 << 23)):
        assert rope(**bad) == mf.EINVAL, bad
    assert rope(positions=0, p=ctypes.byref(mf.pages_t()), cu=0x40) == mf.EINVAL
    assert rope(n=0, q=0, k=0, out_q=0, out_k=0) == mf.OK       # nothing to do


# ---- sanitizers -----------------------------------------------------------------------------------
@needs_toolchain
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                "-Xarch_host", "-fno-sanitize-recover=all"]
    common = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fno-strict-aliasing", f"-I{HEADER}", f"-I{CSRC}"]
    objs = []
    for src in (os.path.join(CSRC, "paged8_api.hip"), os.path.join(SAN, "paged8_stubs.hip")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([HIPCC, *common, *host_san, "-c", src, "-o", objs[-1]])
    objs.append(str(tmp_path / "harness.o"))
    _run([CLANG, "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", f"-I{HEADER}", "-c",
          os.path.join(SAN, "paged8_harness.c"), "-o", objs[-1]])
    exe = str(tmp_path / "paged8_harness")
    _run([HIPCC, "-fsanitize=address,undefined", "-fno-gpu-sanitize", *objs, "-o", exe])
    assert "paged8 harness ok" in _run([exe], env=ENV)


# ---- the oracle itself ------------------------------------------------------------------------------
def test_the_oracles_rounding_is_the_types():
    """Its e4m3 against torch's, its int8 against whole numbers, its exponents against a search."""
    x = torch.cat([torch.randn(5000, dtype=torch.float64) * 2.0 ** i for i in range(-9, 7)]).clamp(-448, 448)
    x = torch.cat([x, torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 448.0, 2.0 ** -6, 0.0624, 17.0, 19.0], dtype=torch.float64)])
    x32 = x.float()
    assert torch.equal(oracle8.rounded(x32.double(), 0, "e4m3"), x32.to(torch.float8_e4m3fn).double())
    y = x32.clamp(-127, 127)
    assert torch.equal(oracle8.rounded(y.double(), 0, "int8"), torch.round(y.double()))
    for code, kind in oracle8.MOST:
        for top in (1.0, 1.75, 1.7500001, 448.0, 449.0, 127.0, 127.01, 3e-5, 1e5, 65504.0):
            e = oracle8.exponent(torch.tensor([top, -top / 2], dtype=torch.float64), code, kind)
            top = min(top, oracle8.MOST[code, kind])
            assert top <= oracle8.TOP[code] * 2.0 ** e and (e == oracle8.LEAST[code, kind] or top > oracle8.TOP[code] * 2.0 ** (e - 1))
