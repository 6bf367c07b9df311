"""Paged attention's weights, ranges and page look-ups where they can go wrong, with inputs whose scores
are exact in fp32: what is left of a weight's error is its exponential's and its roundings'."""
from __future__ import annotations

import pytest
import torch

import paper_2505_22913_amd as mf
from oracle.paged import PagePlan, Refused
from tests.gpu_common import announce
from tests.paged_common import check, fill, starts
from tests.test_gpu_paged import attend

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


# ---- ranges longer than what a wave looks up at once -------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_splits", [1, 2])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 1100), (1500, 4)])
def test_single_tokens_over_ranges_of_many_pages(dtype, d, n_splits, window, sinks):
    """Offsets of 32 tiles of 32 tokens are looked up at once, and again behind them (and behind the sinks')."""
    attend(dtype, 1, 2, d, 16, [1022, 1023, 1024, 1054, 2111, 4999], [1] * 6, window=window, sinks=sinks, n_splits=n_splits, seed=90)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_splits", [1, 2])
@pytest.mark.parametrize("window,sinks", [(0, 0), (5000, 4300), (4500, 4)])
def test_chunks_over_ranges_of_many_pages(dtype, d, n_splits, window, sinks):
    """Offsets of 64 tiles of 64 tokens (32 at d = 256) are looked up at once."""
    attend(dtype, 1, 4, d, 16, [2047, 4095, 4097, 9000], [20, 9, 33, 40], window=window, sinks=sinks, n_splits=n_splits, seed=91)


# ---- the weights' range, and large scores --------------------------------------------------------------
def set_tokens(cache, which, b, x):
    """The tokens x [H][L][d] of request b into its pages."""
    P = cache.page_tokens
    pool = getattr(cache, which)
    for i in range((x.shape[1] + P - 1) // P):
        at = x[:, i * P:(i + 1) * P]
        pool[int(cache.table[b, i]), :, :at.shape[1]] = at.cuda()


def tight(got, q, k, v, scale, dtype, one_part, label, least=0.0):
    """got [n][Hq][d] against float64 where scores are exact in fp32: as in the first test above, with the type's own rounding
    of a weight where it has one part, and `least` for those of its errors that the weight does not scale."""
    n, L, u = q.shape[0], k.shape[1], torch.finfo(dtype).eps / 2
    want, mean = softmax_of(exact_scores(q, k, scale), v, causal(n, L, "cpu"))
    rel = (u if one_part else u * u) + 0.6932 * (2.0 ** -18 + 60 * 2.0 ** -24) + 2.0 ** -22 + (L + 32) * 2.0 ** -24
    tol = half_step(want, dtype) + 2 * rel * mean * (1 + u) + 2 * least
    worst = float(((got.double().cpu() - want).abs() / tol).max())
    announce(f"  {label}: {worst:.2f} of its bound")
    assert worst <= 1, f"{label}: an element is {worst:.2f} of its bound off"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("n_splits", [0, 1])
@pytest.mark.parametrize("late", [False, True])
def test_one_token_26_log2_units_above_the_others(dtype, n, n_splits, late):
    """A token of value 0 whose score is 18 above that of 60000 others: the output is what the others' weights make,
    each 2^-26 of the largest and under fp16's normal numbers. A weight in fp16 is off by up to 2^-25 where the largest is at least
    2^7, 2^-32 of it, whatever the weight."""
    L, d = 60001, 64
    announce(f"peak {dtype} n={n} splits={n_splits} late={late}")
    cache, ks, vs = fill(1, 1, d, 64, [L], dtype, seed=92)
    k, v = torch.zeros_like(ks[0]), (512 + 64 * vs[0].float()).to(dtype)
    j = L - n - 3 if late else 2
    k[0, j], v[0, j] = 2.25, 0.0
    set_tokens(cache, "k", 0, k)
    set_tokens(cache, "v", 0, v)
    q = torch.ones(n, 2, d, dtype=dtype)
    got = mf.mustafar_paged_attn(q.cuda(), cache, starts([n]), n_splits=n_splits, scale=0.125)
    least = L * 2.0 ** -32 * float(v.abs().max()) if dtype == torch.float16 else 0.0
    tight(got, q, k, v, 0.125, dtype, n > 1, "peak", least)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("n_splits", [1, 5])
@pytest.mark.parametrize("high", [16.0, 16384.0])
def test_scores_that_are_large_and_differ_little(dtype, d, n, n_splits, high):
    """Scores of 2^10 or 2^20 with differences of tens, times 2^-5: a common rounding of the softmax's shift takes no part in the
    weights' ratios."""
    L, H, G = 500, 2, 4
    announce(f"large scores {dtype} d={d} n={n} splits={n_splits} high={high}")
    cache, _, vs = fill(1, H, d, 16, [L], dtype, seed=93)
    g = torch.Generator().manual_seed(94)
    k, q = torch.randint(-3, 4, (H, L, d), generator=g).to(dtype), torch.randint(-3, 4, (n, H * G, d), generator=g).to(dtype)
    k[..., 3], q[..., 3] = high, 64.0
    assert float(exact_scores(q, k, 2.0 ** -5).std(-1).max()) < 5
    set_tokens(cache, "k", 0, k)
    got = mf.mustafar_paged_attn(q.cuda(), cache, starts([n]), n_splits=n_splits, scale=2.0 ** -5)
    least = L * 2.0 ** -32 * float(vs[0].abs().max()) if dtype == torch.float16 else 0.0
    tight(got, q, k, vs[0], 2.0 ** -5, dtype, n * G > 16, "large scores", least)


# ---- several layers ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
def test_layers_share_a_steps_table_state_and_stack(dtype):
    """A cache a layer with keys and values of its own; one plan a step, taken on one of them, places every layer's."""
    B, H, G, d, P = 2, 2, 2, 64, 16
    first = mf.PagedCache(B, H, d, 24, P, max_pages=12, dtype=dtype)
    layers = [first] + [mf.PagedCache(B, H, d, 24, P, dtype=dtype, table=first.table, state=first.state, free=first.free)
                        for _ in range(2)]
    held = [[[], []] for _ in layers]
    lens = [0, 0]
    for step, new in enumerate(([40, 17], [1, 1], [30, 1])):
        n = sum(new)
        cu, slots = mf.mustafar_paged_plan(first, torch.tensor(new, dtype=torch.int32, device="cuda"), n)
        lens = [a + b for a, b in zip(lens, new)]
        assert all(c.lens.tolist() == lens for c in layers)
        for layer, (cache, h) in enumerate(zip(layers, held)):
            x = torch.randn(n, (G + 2) * H, d, device="cuda").to(dtype)
            mf.mustafar_paged_write(cache, x[:, G * H:G * H + H], x[:, G * H + H:], slots)
            h[0].append(x[:, G * H:G * H + H].split(new))
            h[1].append(x[:, G * H + H:].split(new))
            out = mf.mustafar_paged_attn(x[:, :G * H], cache, cu, max_q=max(new), max_tokens=max(lens))
            ks, vs = ([torch.cat([p[b] for p in part]).transpose(0, 1) for b in range(B)] for part in h)
            check(out, x[:, :G * H], ks, vs, new, lens, dtype, label=f"step {step} layer {layer}")


# ---- scores that the softmax's shift cannot follow closely ------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 20])
@pytest.mark.parametrize("n_splits", [1, 3])
@pytest.mark.parametrize("bits", [24, 26, 28, 30])
def test_scores_whose_shift_rounds_by_many_bits(dtype, d, n, n_splits, bits):
    """One token far above the others, with scores of 2^24 to 2^30 in which the shift's own rounding is a factor
    of up to 2^64: the output is that token's value, which has the type already."""
    H, G, L = 4, 4, 150
    announce(f"shift {dtype} d={d} n={n} splits={n_splits} bits={bits}")
    cache, ks, vs = fill(1, H, d, 16, [L], dtype, seed=95)
    k = torch.full_like(ks[0], -64.0)
    for h in range(H):
        k[h, 3 + 29 * h] = 64.0
    set_tokens(cache, "k", 0, k)
    g = torch.Generator().manual_seed(96)
    q = (128 + torch.randint(0, 128, (n, H * G, 1), generator=g)).expand(n, H * G, d).to(dtype)     # scores: whole numbers
    got = mf.mustafar_paged_attn(q.contiguous().cuda(), cache, starts([n]), n_splits=n_splits, scale=2.0 ** bits / (128 * 64 * d))
    for h in range(H):
        want = vs[0][h, 3 + 29 * h].expand(n, G, d)
        assert torch.equal(got[:, h * G:(h + 1) * G].cpu(), want), f"kv-head {h}"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("n_splits", [1, 5])
def test_a_range_with_an_infinity_beside_others_at_large_scores(dtype, d, n, n_splits):
    """One channel of one token's value is infinite, so that the rows of its range are done by themselves; scores of 2^20
    times 2^-5 differ by tens, and the other channels get every range's share as closely as without it."""
    L, H, G = 500, 2, 4
    announce(f"infinity at large scores {dtype} d={d} n={n} splits={n_splits}")
    cache, _, vs = fill(1, H, d, 16, [L], dtype, seed=97)
    g = torch.Generator().manual_seed(98)
    k, q = torch.randint(-3, 4, (H, L, d), generator=g).to(dtype), torch.randint(-3, 4, (n, H * G, d), generator=g).to(dtype)
    k[..., 3], q[..., 3] = 16384.0, (64 + torch.arange(H * G) % 7).to(dtype)
    set_tokens(cache, "k", 0, k)
    v = vs[0].clone()
    v[:, 250, 5] = float("inf")
    set_tokens(cache, "v", 0, v)
    got = mf.mustafar_paged_attn(q.cuda(), cache, starts([n]), n_splits=n_splits, scale=2.0 ** -5)
    assert bool((got[..., 5] == float("inf")).all())
    keep = [c for c in range(d) if c != 5]
    score = exact_scores(q, k, 2.0 ** -5)
    want, mean = softmax_of(score, vs[0], causal(n, L, "cpu"))
    u = torch.finfo(dtype).eps / 2
    rel = u + 0.6932 * (2.0 ** -18 + 60 * 2.0 ** -24) + 2.0 ** -22 + (L + 32) * 2.0 ** -24
    if n * G <= 16:
        rel -= u - u * u
    least = L * 2.0 ** -32 * float(vs[0].abs().max()) if dtype == torch.float16 else 0.0
    tol = half_step(want, dtype) + 2 * rel * mean * (1 + u) + 2 * least
    worst = float(((got.double().cpu() - want).abs() / tol)[..., keep].max())
    announce(f"  {worst:.2f} of its bound")
    assert worst <= 1, f"an element is {worst:.2f} of its bound off"


# ---- the binding's numbers -----------------------------------------------------------------------------
@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
@pytest.mark.parametrize("more", [5, 1 << 31, -3, 5 - (1 << 32)])
def test_bounds_and_windows_beyond_32_bits(new, more):
    """A window, first tokens or bounds of 2^32 and some are more than any cache holds, not `some`; negative ones are refused."""
    big = (1 << 32) + more if more > 0 else more
    args = (torch.float16, 2, 2, 64, 16, [300, 20], new)
    for kw in (dict(window=big), dict(window=7, sinks=big), dict(max_q=big), dict(max_tokens=big)):
        if more < 0:
            with pytest.raises(mf.MustafarError):
                attend(*args, **kw)
        else:
            attend(*args, **kw)


# ---- captured ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [90, 1]])
def test_a_captured_call_that_makes_its_own_tensors_replays(dtype, new):
    """Plan, write and attention without status, output and workspace of the caller's, in one graph: every replay gives what eager
    calls on a second cache give, and 0 in the padded rows, with eager work between the replays."""
    B, H, G, d, n = 2, 2, 4, 128, sum(new) + 3
    caches = [fill(B, H, d, 16, [300, 40], dtype, seed=99, spare=60, max_pages=64)[0] for _ in range(2)]
    lens = torch.tensor(new, dtype=torch.int32, device="cuda")
    rows = [torch.randn(n, (G + 2) * H, d, device="cuda").to(dtype) for _ in range(4)]
    x = rows[0].clone()

    def step(cache, x):
        cu, slots = mf.mustafar_paged_plan(cache, lens, n)
        mf.mustafar_paged_write(cache, x[:, H * G:H * (G + 1)], x[:, H * (G + 1):], slots)
        return mf.mustafar_paged_attn(x[:, :H * G], cache, cu, max_q=max(new), max_tokens=900)

    state = caches[0].state.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(caches[0], x)
    assert torch.equal(caches[0].state, state)
    for r in range(4):
        x.copy_(rows[r])
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = step(caches[1], rows[r])
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool((got[-3:] == 0).all()), r
        assert all(c.status.tolist() == [0] for c in caches) and torch.equal(caches[0].state, caches[1].state)


# ---- streams -------------------------------------------------------------------------------------------
def test_plans_and_writes_refuse_a_stream_of_another_device():
    """Before anything is launched or made: tables, state, stack, status and pages stay as they were."""
    class Elsewhere:
        device_index = torch.cuda.current_device() + 1
        cuda_stream = 0
    cache, _, _ = fill(2, 1, 64, 16, [20, 3], torch.float16, seed=99)
    cache.status.fill_(7)
    held = [x.clone() for x in (cache.k, cache.v, cache.table, cache.state, cache.free, cache.status)]
    x, ints = torch.zeros(2, 1, 64, dtype=torch.float16, device="cuda"), lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for call in (lambda: mf.mustafar_paged_plan(cache, ints([1, 1]), 2, stream=Elsewhere()),
                 lambda: mf.mustafar_paged_write(cache, x, x, ints([0, 1]), stream=Elsewhere()),
                 lambda: mf.mustafar_paged_gather(cache, 4, stream=Elsewhere()),
                 lambda: mf.mustafar_paged_attn(x, cache, starts([1, 1]), stream=Elsewhere())):
        with pytest.raises(ValueError, match="stream"):
            call()
    torch.cuda.synchronize()
    for now, was in zip((cache.k, cache.v, cache.table, cache.state, cache.free, cache.status), held):
        assert torch.equal(now, was)
