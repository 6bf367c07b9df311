"""Attention over pages of bfloat16 values near the largest there are: sums of weighted values leave fp32 where their means,
the outputs, do not."""
from __future__ import annotations

import pytest
import torch

import paper_2505_22913_amd as mf
from tests import paged8_common, paged_common
from tests.gpu_common import announce
from tests.paged8_common import CODE, ints, tokens_of
from tests.paged_common import starts

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
MOST = torch.finfo(BF16).max
U = torch.finfo(BF16).eps / 2


def held(kind, ks, vs, P=16):
    """A cache of requests' keys and values (lists of [H][len][d]) in 16 bits or codes, and the values that it holds."""
    B, (H, _, d) = len(ks), ks[0].shape
    lens = [k.shape[1] for k in ks]
    n_pages = sum((n + P - 1) // P for n in lens) + 1
    x = [torch.cat([y.transpose(0, 1) for y in ys]).cuda() for ys in (ks, vs)]
    if kind == "bf16":
        cache = mf.PagedCache(B, H, d, n_pages, P, dtype=BF16)
        _, slots = mf.mustafar_paged_plan(cache, ints(lens), sum(lens))
        mf.mustafar_paged_write(cache, *x, slots)
        return cache, mf.mustafar_paged_attn, paged_common.check, ks, vs
    cache = mf.PagedCache8(B, H, d, n_pages, P, dtype=BF16, code=CODE[kind])
    cu, _ = mf.mustafar_paged_plan(cache, ints(lens), sum(lens))
    mf.mustafar_paged8_write(cache, *x, cu)
    now = [[tokens_of(cache, w, b).to(BF16).cpu() for b in range(B)] for w in ("k", "v")]
    return cache, mf.mustafar_paged8_attn, paged8_common.check, *now


def large(H, n, d, g):
    """Values of which a channel has the largest there is, of one sign or both, in every token or in two, beside ordinary ones."""
    v = torch.randn(H, n, d, generator=g)
    v[..., 0::8] = MOST
    v[..., 1::8] = -MOST
    v[..., 2::8] = torch.where(v[..., 2::8] > 0, MOST, -MOST)
    v[:, [0, n // 2], 4::8] = MOST
    v[..., 5::8] *= 2.0 ** 122
    return v.to(BF16)


# as many ranges, more than a wave's weights, and shared out by the lengths (8-bit codes)
SPLITS = [dict(n_splits=1), dict(n_splits=5), dict(n_splits=70), dict(max_tokens=300000)]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [70, 1, 33, 2]])
@pytest.mark.parametrize("hints", SPLITS)
@pytest.mark.parametrize("spread", [0.0, 1.0])
def test_means_of_the_largest_values_are_finite(kind, d, new, hints, spread):
    """Every output is a mean of values, so none is infinite; in 16 bits one channel holds an infinity, which stays in it."""
    H, G, lens = 2, 4, [500, 40, 33, 2]
    announce(f"largest {kind} d={d} new={new} {hints} spread={spread}")
    g = torch.Generator().manual_seed(d)
    ks, vs = [torch.randn(H, n, d, generator=g).to(BF16) for n in lens], [large(H, n, d, g) for n in lens]
    vs[0][:, 20, 7] = float("inf")
    cache, attn, check, ks, vs = held(kind, ks, vs)
    q = (torch.randn(sum(new), H * G, d, generator=g) * spread).to(BF16).cuda()
    got = attn(q, cache, starts(new), **hints)
    check(got, q, ks, vs, new, lens, BF16, label="largest")
    again = attn(q, cache, starts(new), **hints)
    assert torch.equal(got.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("n_splits", [3, 5, 12, 70])
def test_ranges_that_are_finite_by_themselves(kind, d, n, n_splits):
    """Sums of a range's weighted values that fp32 holds, and of all ranges' that it does not: a weight is 2^7 where scores
    are equal, so a range of L / n_splits tokens of 2^114 and the like reaches 2^127, all of them 2^128 and more."""
    L, H, G = 100 * n_splits, 1, 2
    announce(f"ranges {kind} d={d} n={n} splits={n_splits}")
    g = torch.Generator().manual_seed(n + d)
    v = torch.randn(H, L, d, generator=g)
    v[..., ::2] = 1.9375 * 2.0 ** 113
    cache, attn, check, ks, vs = held(kind, [torch.randn(H, L, d, generator=g).to(BF16)], [v.to(BF16)])
    q = torch.zeros(n, H * G, d, dtype=BF16, device="cuda")
    check(attn(q, cache, starts([n]), n_splits=n_splits), q, ks, vs, [n], [L], BF16, label="ranges")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 20])
@pytest.mark.parametrize("n_splits", [1, 3, 20])
@pytest.mark.parametrize("bits", [0, 23, 26, 28, 29, 30, 33])
def test_equal_scores_of_any_size(d, n, n_splits, bits):
    """Equal scores up to 2^33, exact in fp32, so that the weights are equal and outputs the values' mean: of the largest values in one
    half of the tokens (some ranges have none) as of ordinary and of the smallest ones beside them.

    A sum of L values is off by L 2^-24 of their magnitudes', its factors by as little."""
    H, G, L = 1, 2, 300
    announce(f"equal scores d={d} n={n} splits={n_splits} bits={bits}")
    g = torch.Generator().manual_seed(bits)
    v = torch.randn(H, L, d, generator=g)
    v[..., 0::4] = MOST
    v[:, :L // 2, 1::4] = -MOST
    v[..., 2::4] *= 2.0 ** -110
    cache, attn, _, ks, vs = held("bf16", [torch.full((H, L, d), 64.0).to(BF16)], [v.to(BF16)])
    q = torch.full((n, H * G, d), 128.0, dtype=BF16, device="cuda")
    got = attn(q, cache, starts([n]), n_splits=n_splits, scale=2.0 ** bits / (128 * 64 * d)).double().cpu()
    for i in range(n):
        x = vs[0][0, :L - n + 1 + i].double()
        tol = U * x.mean(0).abs() + 2 * (L + 32) * 2.0 ** -24 * x.abs().mean(0) * (1 + U)
        worst = ((got[i] - x.mean(0)).abs() / tol).amax(0)
        assert float(worst.max()) <= 1, f"row {i}: {[float(worst[c::4].max()) for c in range(4)]} of the bound, by channel"


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 1, 1], [33, 1, 5]])
@pytest.mark.parametrize("hints", SPLITS)
@pytest.mark.parametrize("sign", [-1.0, 1.0, 0.0])
def test_large_queries_over_small_keys(kind, d, new, hints, sign):
    """A query's channel of 2^122 over keys of 2^-104, whose codes' sums alone leave fp32: scores of one sign or both, around 1 by a scale
    of 2^-18; the other channels' products are under 2^-100 of that."""
    H, G, lens = 2, 2, [400, 40, 9]
    announce(f"large queries {kind} d={d} new={new} {hints} sign={sign}")
    g = torch.Generator().manual_seed(d)
    ks, vs = [[torch.randn(H, n, d, generator=g) for n in lens] for _ in range(2)]
    for k in ks:
        k *= 2.0 ** -105
        if sign:
            k[..., 3] = sign * k[..., 3].abs()
    cache, attn, check, ks, vs = held(kind, [k.to(BF16) for k in ks], [v.to(BF16) for v in vs])
    q = torch.randn(sum(new), H * G, d, generator=g)
    q[..., 3] = 2.0 ** 122
    q = q.to(BF16).cuda()
    check(attn(q, cache, starts(new), scale=2.0 ** -18, **hints), q, ks, vs, new, lens, BF16, scale=2.0 ** -18, label="large queries")
