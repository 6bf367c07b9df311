"""Helpers of the 8-bit paged cache's tests: filled caches, and their values."""
from __future__ import annotations

import torch

import paper_2505_22913_amd as mf
from oracle import paged as oracle_paged
from tests.paged_common import bound

KIND = {torch.float16: "fp16", torch.bfloat16: "bf16"}
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def values_of(codes, scale):
    """Codes [..][P][d] and their scale bytes [..][P / block] as float64."""
    power = torch.tensor([2.0 ** (i - 127) for i in range(256)], dtype=torch.float64, device=scale.device)[scale.long()]
    return codes.double() * power.repeat_interleave(codes.shape[-2] // scale.shape[-1], -1)[..., None]


def tokens_of(cache, which, b):
    """The values of request b's tokens, float64 [H][len][d]."""
    codes, scale = (cache.k, cache.k_scale) if which == "k" else (cache.v, cache.v_scale)
    n, P = int(cache.lens[b]), cache.page_tokens
    pages = cache.table[b, :(n + P - 1) // P].long()
    x = values_of(codes.view(torch.uint8)[pages].view(codes.dtype), scale[pages])          # [pages][H][P][d]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def fill8(B, H, d, P, lens, dtype, code, block, seed=0, spare=3, layout="heads", junk=None, k_scale=0, v_scale=0, max_pages=None):
    """A PagedCache8 of random codes in scattered pages whose blocks have random exponents (around 2^-5 for e4m3 and
    2^-6 for int8, plus k_scale and v_scale), and the tokens' values: lists of [H][len][d] of the type. junk: what the
    other tokens' codes are (None: random) with blocks of exponent byte 255 where no token is."""
    g = torch.Generator().manual_seed(seed)
    blocks = [(n + P - 1) // P for n in lens]
    n_pages = sum(blocks) + spare
    max_pages = max(max(blocks), 1) + 1 if max_pages is None else max_pages
    order = torch.randperm(n_pages, generator=g).tolist()
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    used = torch.zeros(n_pages, P, dtype=torch.bool)
    for b, n in enumerate(lens):
        for i in range(blocks[b]):
            table[b, i] = order[at]
            used[order[at], :min(P, n - i * P)] = True
            at += 1
    pools, scales = [], []
    for extra in (k_scale, v_scale):
        x = torch.randn(n_pages, H, P, d, generator=g)
        x = (x * 30).to(torch.float8_e4m3fn).view(torch.uint8) if code == "e4m3" else (x * 40).round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
        if junk is not None:
            x = torch.where(used[:, None, :, None], x, junk)
        byte = torch.randint(0, 3, (n_pages, H, P // block), generator=g) + 127 - (6 if code == "e4m3" else 7) + extra
        if junk is not None:
            byte = torch.where(used.view(n_pages, 1, P // block, block).any(-1), byte, 255)
        x = x if layout == "heads" else x.transpose(1, 2).contiguous().transpose(1, 2)
        on = x.cuda() if layout == "heads" else x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        pools.append(on.view(CODE[code]))
        scales.append(byte.to(torch.uint8).cuda())
    state = torch.tensor(list(lens) + [n_pages - at, 0], dtype=torch.int32)
    free = torch.zeros(n_pages, dtype=torch.int32)
    free[:n_pages - at] = torch.tensor(order[at:], dtype=torch.int32)
    cache = mf.PagedCache8(B, H, d, n_pages, P, dtype=dtype, block_tokens=block, k=pools[0], v=pools[1], k_scale=scales[0],
                           v_scale=scales[1], table=table.cuda(), state=state.cuda(), free=free.cuda())
    out = []
    for which in ("k", "v"):
        xs = [tokens_of(cache, which, b) for b in range(B)]
        for x in xs:
            assert torch.equal(x.to(dtype).double().nan_to_num(7.0), x.nan_to_num(7.0))     # values of the type
        out.append([x.to(dtype) for x in xs])
    return cache, out[0], out[1]


def check(got, q, ks, vs, new, lens, dtype, window=0, sinks=0, scale=None, label=""):
    """As paged_common.check, for values that may be 0 where the weight is: bound() is a multiple of the output and of
    the weighted mean of |v|, and fp16 has two errors that are not. Its numbers under 2^-14 are multiples of 2^-24, so an output's
    rounding is up to 2^-25 whatever its size; and a row's weights are multiples of 2^-24 where the largest is at least 2^7, so each
    of its n weights is up to 2^-32 of that off, which |v| multiplies. (bf16 has fp32's exponents.)"""
    u, at, worst, d = torch.finfo(dtype).eps / 2, 0, 0.0, q.shape[2]
    G = q.shape[1] // ks[0].shape[0]
    for b, (n, L) in enumerate(zip(new, lens)):
        m = min(n, L)      # rows before the request's first token see nothing
        lead, rows = got[at:at + n - m], got[at + n - m:at + n].double()
        assert bool((lead == 0).all()), f"{label}: request {b}: a row that sees nothing is not 0"
        if m:
            want, mean, mag = oracle_paged.attention(q[at + n - m:at + n], ks[b].to(q.device), vs[b].to(q.device), m, window, sinks,
                                                     scale)
            fine = torch.isfinite(want)
            assert torch.equal(torch.isnan(rows), torch.isnan(want)), f"{label}: request {b}: NaN elsewhere"
            odd = ~fine & ~torch.isnan(want)
            assert torch.equal(rows[odd], want[odd]), f"{label}: request {b}: infinities elsewhere"
            err = torch.where(fine, (rows - want).abs(), 0.0)
            tol = bound(torch.where(fine, want, 0.0), mean, mag, L, d, dtype)
            least = 0.0
            if dtype == torch.float16:
                most_v = vs[b].to(q.device).double().nan_to_num(0.0).abs().amax(1).repeat_interleave(G, 0)      # [Hq][d]
                least = 2.0 ** -25 + L * 2.0 ** -32 * most_v
            tol = tol + least
            ratio = float(torch.where(fine, err / tol, 0.0).max())
            rel = float(torch.where(fine, (err - least).clamp(min=0), 0.0).norm() / torch.where(fine, want, 0.0).norm().clamp(min=1e-30))
            most = 2 * u + float(mag.max()) * 4 * d * 2.0 ** -24
            worst = max(worst, rel / u)
            assert ratio <= 1, f"{label}: request {b} ({n} of {L} tokens): an element is {ratio:.2f} of its bound off"
            assert rel <= most, f"{label}: request {b} ({n} of {L} tokens): 2-norm {rel:.2e} of {most:.2e}"
        at += n
    return worst
