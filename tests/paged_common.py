"""Helpers of the paged cache's tests: filled caches, and the error that attention may have."""
from __future__ import annotations

import torch

import paper_2505_22913_amd as mf
from oracle import paged as oracle_paged

LN2 = 0.6931471805599453


def fill(B, H, d, P, lens, dtype=torch.float16, seed=0, spare=3, layout="heads", junk=None, k_scale=1.0, max_pages=None):
    """A PagedCache holding random tokens in scattered pages, and the tokens: lists of [H][len][d]."""
    g = torch.Generator().manual_seed(seed)
    blocks = [(n + P - 1) // P for n in lens]
    n_pages = sum(blocks) + spare
    max_pages = max(max(blocks), 1) + 1 if max_pages is None else max_pages
    ks = [(torch.randn(H, n, d, generator=g) * k_scale).to(dtype) for n in lens]
    vs = [torch.randn(H, n, d, generator=g).to(dtype) for n in lens]
    order = torch.randperm(n_pages, generator=g).tolist()
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    pools = []
    for _ in range(2):
        shape = (n_pages, H, P, d) if layout == "heads" else (n_pages, P, H, d)
        x = torch.randn(shape, generator=g).to(dtype) if junk is None else torch.full(shape, junk, dtype=dtype)
        pools.append(x if layout == "heads" else x.transpose(1, 2))
    at = 0
    for b, n in enumerate(lens):
        for i in range(blocks[b]):
            page = order[at]
            at += 1
            table[b, i] = page
            m = min(P, n - i * P)
            for pool, x in zip(pools, (ks[b], vs[b])):
                pool[page, :, :m] = x[:, i * P:i * P + m]
    state = torch.tensor(list(lens) + [n_pages - at, 0], dtype=torch.int32)
    free = torch.zeros(n_pages, dtype=torch.int32)
    free[:n_pages - at] = torch.tensor(order[at:], dtype=torch.int32)
    pools = [p.cuda() if layout == "heads" else p.transpose(1, 2).contiguous().cuda().transpose(1, 2) for p in pools]
    cache = mf.PagedCache(B, H, d, n_pages, P, k=pools[0], v=pools[1], table=table.cuda(), state=state.cuda(),
                          free=free.cuda())
    return cache, ks, vs


def starts(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def bound(out, mean, mag, n, d, dtype):
    """Largest error of an output element, from the roundings that the kernels make:
    u = half a step of the type. The output is rounded once (u |out|). Each weight is off by its own rounding
    (u), by its score's, an fp32 sum of d products (mag 2 d 2^-24 at most, the maximum's
    too) in the exponent, and by exp2 and the sums over n weights (n + 32 steps of 2^-24); the normalised weights by twice
    that; their errors are multiplied by |v|, mean = sum of weights times |v|."""
    u = torch.finfo(dtype).eps / 2
    weight = u + mag[..., None] * 4 * d * 2.0 ** -24 + (n + 32) * 2.0 ** -24
    return u * out.abs() + 2 * weight * mean * (1 + u) + 1e-30


def check(got, q, ks, vs, new, lens, dtype, window=0, sinks=0, scale=None, label=""):
    """got [n_q][Hq][d] against float64, request by request: every element within bound(), and the 2-norm of
    the error within 2 u of the output's plus what the scores' errors make (independent roundings of weights and
    output, of rms u / sqrt(3) each at most, add up to 0.82 u)."""
    u, at, worst, d = torch.finfo(dtype).eps / 2, 0, 0.0, q.shape[2]
    for b, (n, L) in enumerate(zip(new, lens)):
        if n == 0:
            continue
        m = min(n, L)      # rows before the request's first token see nothing
        lead, rows = got[at:at + n - m], got[at + n - m:at + n].double()
        assert bool((lead == 0).all()), f"{label}: request {b}: a row that sees nothing is not 0"
        if m:
            want, mean, mag = oracle_paged.attention(q[at + n - m:at + n], ks[b].to(q.device), vs[b].to(q.device), m, window,
                                                     sinks, scale)
            fine = torch.isfinite(want)
            assert torch.equal(torch.isnan(rows), torch.isnan(want)), f"{label}: request {b}: NaN elsewhere"
            odd = ~fine & ~torch.isnan(want)
            assert torch.equal(rows[odd], want[odd]), f"{label}: request {b}: infinities elsewhere"
            err = torch.where(fine, (rows - want).abs(), 0.0)
            tol = bound(torch.where(fine, want, 0.0), mean, mag, L, d, dtype)
            ratio = float(torch.where(fine, err / tol, 0.0).max())
            rel = float(err.norm() / torch.where(fine, want, 0.0).norm().clamp(min=1e-30))
            most = 2 * u + float(mag.max()) * 4 * d * 2.0 ** -24
            worst = max(worst, rel / u)
            assert ratio <= 1, f"{label}: request {b} ({n} of {L} tokens): an element is {ratio:.2f} of its bound off"
            assert rel <= most, f"{label}: request {b} ({n} of {L} tokens): 2-norm {rel:.2e} of {most:.2e}"
        at += n
    return worst
