"""Paged attention's weights, ranges and page look-ups where they can go wrong, with inputs whose scores
are exact in fp32: what is left of a weight's error is its exponential's and its roundings'."""
from __future__ import annotations

import pytest
import torch

import paper_2505_22913_amd as mf
from oracle.paged import PagePlan, Refused
from tests.gpu_common import announce
from tests.paged_common import check, fill, starts

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


def half_step(x, dtype):
    """Half the distance of the type's numbers at |x| (float64)."""
    eps = torch.finfo(dtype).eps
    least = torch.finfo(dtype).tiny
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=least)))) * eps / 2


def exact_scores(q, k, scale):
    """The scores of q [n][Hq][d] and k [H][L][d] whose entries are small whole numbers, float64 [Hq][n][L]."""
    G = q.shape[1] // k.shape[0]
    return q.double().transpose(0, 1) @ k.double().repeat_interleave(G, 0).transpose(1, 2) * scale


def softmax_of(score, v, sees):
    """Output and the weights' mean of |v|, float64 [n][Hq][d]."""
    G = score.shape[0] // v.shape[0]
    p = torch.softmax(score.masked_fill(~sees, -torch.inf), -1)
    v = v.double().repeat_interleave(G, 0)
    return (p @ v).transpose(0, 1), (p @ v.abs()).transpose(0, 1)


def causal(n, L, device):
    return torch.arange(L, device=device)[None] <= torch.arange(L - n, L, device=device)[:, None]


# ---- the weights' precision ----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(4, 1), (2, 4), (1, 16)])
@pytest.mark.parametrize("n_splits", [1, 5])
def test_single_tokens_weights_are_not_rounded_to_the_type(dtype, d, H, G, n_splits):
    """Tokens whose output is off by no more than its own rounding and what 2 parts of the type leave of the weights.

    q and k are whole numbers up to 3, so every score is exact in fp32. A weight 2^x, x up to 60 in magnitude, is off by
    ln 2 (2^-18 + 60 2^-24) from x's last rounding and the scale's, 2^-22 from the exponential, and from its two parts by u^2
    (u = half a step of the type; of fp16 also 2^-25 where the reference's is 2^7). The sums over the tokens add (n + 32) 2^-24, and the
    normalised weights are off by twice all that."""
    L, n = 700, 1
    scale = 2.0 ** -5
    announce(f"weights {dtype} d={d} H={H} G={G} splits={n_splits}")
    cache, ks, vs = fill(3, H, d, 16, [L, 33, 1], dtype, seed=d + G)
    g = torch.Generator().manual_seed(d)
    for b, m in enumerate((L, 33, 1)):
        ks[b] = torch.randint(-3, 4, (H, m, d), generator=g).to(dtype)
        for i in range((m + 15) // 16):
            at = ks[b][:, 16 * i:16 * i + 16]
            cache.k[int(cache.table[b, i]), :, :at.shape[1]] = at.cuda()
    q = torch.randint(-3, 4, (3, H * G, d), generator=g).to(dtype)
    got = mf.mustafar_paged_attn(q.cuda(), cache, starts([1, 1, 1]), scale=scale, n_splits=n_splits).double().cpu()
    u = torch.finfo(dtype).eps / 2
    for b, m in enumerate((L, 33, 1)):
        score = exact_scores(q[b:b + 1], ks[b], scale)
        assert float(score.abs().max()) < 40 * 0.69
        want, mean = softmax_of(score, vs[b], causal(n, m, "cpu"))
        rel = 0.6932 * (2.0 ** -18 + 60 * 2.0 ** -24) + 2.0 ** -22 + u * u + (m + 32) * 2.0 ** -24
        least = m * 2.0 ** -32 * float(vs[b].abs().max()) if dtype == torch.float16 else 0.0
        tol = half_step(want, dtype) + 2 * rel * mean * (1 + u) + 2 * least
        err = (got[b:b + 1] - want).abs()
        worst = float((err / tol).max())
        over = float(((err - half_step(want, dtype)) / (mean * u)).max())
        announce(f"  request {b}: {worst:.2f} of its bound; beyond the output's rounding {over:.4f} u mean |v|")
        assert worst <= 1, f"request {b}: an element is {worst:.2f} of its bound off"


# ---- plans ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_slots", [4, 5000])
@pytest.mark.parametrize("lens,n_free,keep,new", [
    ([64, 30], 30, [0, 0], [0, 0]),             # every page is on the stack and six of them are in tables: nothing may go on it
    ([64, 30], 25, [0, 30], [0, 1]),            # one page too many
    ([64, 30], 30, None, [1, 1]),               # nothing is given up, but what is taken is held already
    ([480, 16], 0, [0, 0], [1, 1]),
])
def test_a_plan_of_more_pages_than_there_are_is_refused(lens, n_free, keep, new, n_slots):
    """A state whose tables and stack hold more pages than the pool has: the stack has no room for those given up."""
    n_pages, guard = 30, 64
    free = torch.full((n_pages + guard,), -7, dtype=torch.int32, device="cuda")
    free[:n_pages] = torch.arange(n_pages - 1, -1, -1, device="cuda")
    cache = mf.PagedCache(2, 1, 64, n_pages, 16, max_pages=40, free=free[:n_pages],
                          state=torch.tensor(lens + [n_free, 0], dtype=torch.int32, device="cuda"))
    before = [x.clone() for x in (free, cache.table, cache.state)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    status = ints([0])
    cu, slots = mf.mustafar_paged_plan(cache, ints(new), n_slots, keep=None if keep is None else ints(keep), status=status)
    assert status.tolist() == [mf.PLAN_STATE] and cu.tolist() == [0, 0, 0] and bool((slots == -1).all())
    for x, y in zip(before, (free, cache.table, cache.state)):
        assert torch.equal(x, y)
    plan = PagePlan(2, 16, n_pages, 40)
    plan.lens, plan.tables, plan.stack = lens, [list(range((n + 15) // 16)) for n in lens], list(range(n_free))
    with pytest.raises(Refused) as e:
        plan.step(new, keep, n_slots)
    assert e.value.args == (mf.PLAN_STATE,)


# ---- the workspace of calls of both kinds -----------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 300, 0, 2], [1, 1, 1, 6], [1] * 30 + [9]])
@pytest.mark.parametrize("n_splits", [0, 2, 9, 70])
@pytest.mark.parametrize("bad", [None, float("inf")])
def test_ranges_of_single_tokens_lie_inside_the_workspace(dtype, d, new, n_splits, bad):
    """Single tokens beside chunks, few rows of which make the entries' rows the smaller ones or q's: a workspace of
    exactly what is asked for, of NaN, between guards; with a value that every row sees infinite in two requests."""
    cached = [(700, 50, 3, 90)[b % 4] for b in range(len(new))]
    lens = [a + b for a, b in zip(cached, new)]
    announce(f"workspace {dtype} d={d} new={new} splits={n_splits} bad={bad}")
    cache, ks, vs = fill(len(new), 2, d, 16, lens, dtype, seed=70)
    if bad is not None:
        for b in (0, 1):
            cache.v[int(cache.table[b, 0]), 1, 2, 7] = bad
            vs[b][1, 2, 7] = bad
    g = torch.Generator().manual_seed(71)
    q = torch.randn(sum(new), 8, d, generator=g).to(dtype).cuda()
    need = mf.mustafar_paged_attn_workspace_bytes(cache, 8, sum(new), max(new), 900, n_splits)
    assert need > 0
    whole = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    got = mf.mustafar_paged_attn(q, cache, starts(new), max_q=max(new), max_tokens=900, n_splits=n_splits, ws=whole[256:256 + need])
    check(got, q, ks, vs, new, lens, dtype, label="workspace")
    assert bool((whole[:256] == 255).all()) and bool((whole[256 + need:] == 255).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [200, 90]])
def test_a_refused_step_is_told_and_gives_no_memory_of_others(dtype, new):
    """Too few pages: the cache's status says so, the write leaves the pages as they are and attention's output is 0;
    after pages have been given back the same step is taken, and the status is 0 again."""
    lens, d = [48, 64], 128
    cache, ks, vs = fill(2, 2, d, 16, lens, dtype, seed=80, spare=0, max_pages=40)
    assert cache.status.tolist() == [0]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    n = sum(new)
    x = torch.randn(n, 2, d, device="cuda").to(dtype)
    q = torch.randn(n, 8, d, device="cuda").to(dtype)
    before = [t.clone() for t in (cache.k, cache.v, cache.state, cache.table)]
    cu, slots = mf.mustafar_paged_plan(cache, ints([1, 1] if new == [1, 1] else new), n)
    mf.mustafar_paged_write(cache, x, x, slots)
    for _ in range(4):
        dirty = [torch.full_like(q, float("nan")) for _ in range(8)]     # what the allocator hands out next
        torch.cuda.synchronize()
        del dirty
        out = mf.mustafar_paged_attn(q, cache, cu, max_q=max(new), max_tokens=300)
        assert bool((out == 0).all())
    assert cache.status.tolist() == [mf.PLAN_PAGES]
    for t, y in zip(before, (cache.k, cache.v, cache.state, cache.table)):
        assert torch.equal(t, y)
    mf.mustafar_paged_plan(cache, ints([0, 0]), 0, keep=ints([48, 10]))
    assert cache.status.tolist() == [0]
    cu, slots = mf.mustafar_paged_plan(cache, ints([1, 0]), 3)           # padded: rows behind the last are 0 too
    assert cache.status.tolist() == [0] and cu.tolist() == [0, 1, 1]
    mf.mustafar_paged_write(cache, x[:1].expand(3, 2, d).contiguous(), x[:1].expand(3, 2, d).contiguous(), slots)
    dirty = torch.full((3, 8, d), float("nan"), dtype=dtype, device="cuda")
    del dirty
    out = mf.mustafar_paged_attn(q[:1].expand(3, 8, d).contiguous(), cache, cu, max_q=1, max_tokens=300)
    new_k = [torch.cat([t[0], x[:1].cpu().transpose(0, 1)], 1) for t in (ks, vs)]
    check(out[:1], q[:1], [new_k[0]], [new_k[1]], [1], [49], dtype, label="padded")
    assert bool((out[1:] == 0).all())
    torch.cuda.synchronize()
    own = ints([5])
    mf.mustafar_paged_plan(cache, ints([1000, 0]), 2000, status=own)     # a status of the call's own
    assert own.tolist() == [mf.PLAN_TABLE] and cache.status.tolist() == [0]
