"""The paged dense cache on the GPU: plans, writes, gathers and attention against plain
computations, and a serving loop of them together with the compressed caches."""
import random

import numpy as np
import pytest
import torch

import oracle
import paper_2505_22913_amd as mf
from oracle.paged import PagePlan, Refused
from tests.gpu_common import ATTN_TOL, announce, attn_error
from tests.paged_common import check, fill, starts

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- plans -------------------------------------------------------------------------------------
def same_plan(cache, plan, cu, slots, want):
    assert cu.tolist() == want[0]
    assert slots.tolist() == want[1]
    state = cache.state.tolist()
    assert state[:-2] == plan.lens and state[-2] == len(plan.stack) and state[-1] == 0
    free, table = cache.free.tolist(), cache.table.tolist()
    assert free[:len(plan.stack)] == plan.stack
    assert [row[:len(t)] for row, t in zip(table, plan.tables)] == plan.tables


@pytest.mark.parametrize("B,P,most_new,n_slots", [(1, 16, 40, 64), (3, 64, 200, 700), (64, 16, 90, 6000),
                                                  (257, 32, 30, 9000), (4096, 16, 3, 13000), (5, 1024, 3000, 15000)])
@pytest.mark.parametrize("aside", [False, True])
def test_plans_follow_the_lengths(B, P, most_new, n_slots, aside):
    """Steps that add tokens, take some back and replace requests, in place and into another state."""
    rng = random.Random(B + P + aside)
    n_pages = B * (3 * most_new // P + 2)
    plan = PagePlan(B, P, n_pages, 4 * most_new // P + 3)
    cache = mf.PagedCache(B, 1, 64, n_pages, P, max_pages=plan.max_pages)
    states = [cache.state, torch.zeros_like(cache.state)]
    for i in range(7):
        announce(f"plan B={B} P={P} aside={aside} step {i}")
        new = [rng.choice([0, 1, 1, rng.randint(0, most_new)]) for _ in range(B)]
        keep = None
        if i % 2:
            keep = [rng.choice([n, n, 0, rng.randint(-2, n + 5)]) if n < 2 * most_new else 0 for n in plan.lens]
        elif i:
            keep = [n if n < 2 * most_new else 0 for n in plan.lens]
        status = ints([77])
        before = cache.state.clone()
        out = states[(i + 1) % 2] if aside else None
        cu, slots = mf.mustafar_paged_plan(cache, ints(new), n_slots, keep=None if keep is None else ints(keep),
                                           state_out=out, status=status)
        want = plan.step(new, keep, n_slots)
        assert status.tolist() == [0]
        if aside:
            assert torch.equal(cache.state, before)
            cache = mf.PagedCache(B, 1, 64, n_pages, P, k=cache.k, v=cache.v, table=cache.table, state=out, free=cache.free)
        same_plan(cache, plan, cu, slots, want)


def test_a_step_taken_back_leaves_the_stack_as_it_was():
    plan_lens = [5, 64, 130, 0]
    cache = mf.PagedCache(4, 1, 64, 40, 16, max_pages=20)
    mf.mustafar_paged_plan(cache, ints(plan_lens), 300)
    free, state, table = cache.free.clone(), cache.state.clone(), cache.table.clone()
    mf.mustafar_paged_plan(cache, ints([40, 1, 33, 17]), 300)
    assert cache.lens.tolist() == [45, 65, 163, 17]
    mf.mustafar_paged_plan(cache, ints([0, 0, 0, 0]), 300, keep=ints(plan_lens))
    n = state[4]
    assert torch.equal(cache.state, state) and torch.equal(cache.free[:n], free[:n])
    for b, L in enumerate(plan_lens):
        assert torch.equal(cache.table[b, :(L + 15) // 16], table[b, :(L + 15) // 16])


@pytest.mark.parametrize("new,n_slots,why", [([600, 0], 1000, mf.PLAN_PAGES), ([200, 200], 399, mf.PLAN_SLOTS),
                                             ([700, 1], 1000, mf.PLAN_TABLE), ([-1, 4], 1000, mf.PLAN_STATE),
                                             ([2000000000, 1], 1000, mf.PLAN_TABLE | mf.PLAN_SLOTS),
                                             ([-2147483648, 900], 1000, mf.PLAN_STATE | mf.PLAN_TABLE)])
@pytest.mark.parametrize("many", [False, True])
def test_a_plan_that_cannot_be_taken_changes_nothing(new, n_slots, why, many):
    n_slots += 4096 * many if why not in (mf.PLAN_SLOTS,) else 0      # several workgroups
    cache = mf.PagedCache(2, 1, 64, 30, 16, max_pages=40)
    mf.mustafar_paged_plan(cache, ints([20, 1]), 64)
    before = [x.clone() for x in (cache.table, cache.free, cache.state)]
    status = ints([0])
    cu, slots = mf.mustafar_paged_plan(cache, ints(new), n_slots, status=status)
    assert status.tolist() == [why]
    assert cu.tolist() == [0, 0, 0] and bool((slots == -1).all())
    for x, y in zip(before, (cache.table, cache.free, cache.state)):
        assert torch.equal(x, y)
    plan = PagePlan(2, 16, 30, 40)
    plan.step([20, 1])
    with pytest.raises(Refused) as e:
        plan.step(new, None, n_slots)
    assert e.value.args == (why,)


def test_a_plan_of_a_state_that_is_none_is_refused():
    cache = mf.PagedCache(2, 1, 64, 30, 16, max_pages=4)
    for bad in ([-5, 3, 10, 0], [65, 3, 10, 0], [3, 3, 31, 0], [3, 3, -1, 0]):
        cache.state.copy_(ints(bad))
        status = ints([0])
        mf.mustafar_paged_plan(cache, ints([1, 1]), 2, status=status)
        assert status.tolist() == [mf.PLAN_STATE] and cache.state.tolist() == bad


# ---- writes and gathers ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("H,d,P,n,packed", [(1, 64, 16, 1, False), (8, 128, 64, 257, True), (3, 256, 32, 100, False),
                                            (32, 128, 16, 1000, True)])
def test_tokens_are_written_to_their_slots(dtype, layout, H, d, P, n, packed):
    cache, _, _ = fill(1, H, d, P, [n + 50], dtype, seed=n, layout=layout)
    n_pages = cache.desc.n_pages
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, 2 * H + 3 if packed else 2 * H, d, generator=g).to(dtype).cuda()
    k_new, v_new = x[:, :H], x[:, H:2 * H]
    slots = torch.randperm(n_pages * P, generator=g)[:n].int()
    slots[::7] = -1
    slots[3::11] = n_pages * P + 5      # outside: left out
    want = [p.clone() for p in (cache.k, cache.v)]
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * P:
            want[0][s // P, :, s % P], want[1][s // P, :, s % P] = k_new[t], v_new[t]
    mf.mustafar_paged_write(cache, k_new, v_new, slots.cuda())
    assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("H,d,P,lens,first,n_max", [(1, 64, 16, [1], None, 1), (4, 128, 64, [200, 0, 64, 1], None, 131),
                                                    (2, 256, 32, [100, 33], [7, 33], 70), (3, 128, 1024, [1500], [1023], 600)])
def test_pages_are_gathered(dtype, layout, H, d, P, lens, first, n_max):
    B = len(lens)
    cache, ks, vs = fill(B, H, d, P, lens, dtype, seed=d, layout=layout)
    x_k, x_v = (torch.full((B, H, n_max, d), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    mf.mustafar_paged_gather(cache, n_max, first=None if first is None else ints(first), x_k=x_k, x_v=x_v)
    for got, xs in ((x_k, ks), (x_v, vs)):
        for b, n in enumerate(lens):
            f = first[b] if first else 0
            m = max(0, min(n - f, n_max))
            assert torch.equal(got[b, :, :m].cpu(), xs[b][:, f:f + m].float().half())
            assert bool((got[b, :, m:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_outputs_larger_than_the_caches_are_gathered(dtype):
    B, H, d, P, n_max = 2, 8, 128, 64, 35001       # 287 MB
    lens, first = [35100, 20], [98, 0]
    cache = mf.PagedCache(B, H, d, 560, P, max_pages=552, dtype=dtype)
    cache.k.normal_()
    cache.v.normal_()
    mf.mustafar_paged_plan(cache, ints(lens), sum(lens))
    x = [torch.full((B, H, n_max, d), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    mf.mustafar_paged_gather(cache, n_max, first=ints(first), x_k=x[0], x_v=x[1])
    for got, pool in zip(x, (cache.k, cache.v)):
        for b, (n, f) in enumerate(zip(lens, first)):
            m = min(n - f, n_max)
            pages = cache.table[b, :(n + P - 1) // P].long()
            want = pool[pages].transpose(0, 1).reshape(H, -1, d)[:, f:f + m].half()
            assert torch.equal(got[b, :, :m], want) and bool((got[b, :, m:] == 7).all())


def test_bf16_values_beyond_fp16_are_gathered_as_its_largest():
    cache, _, _ = fill(1, 1, 64, 16, [16], torch.bfloat16)
    row = torch.tensor([1e5, -1e5, 3e38, float("inf"), -float("inf"), float("nan"), 65504.0, 65280.0, 1e-8, -1e-6] + [0.5] * 54)
    cache.k[cache.table[0, 0], 0, 3] = row.bfloat16().cuda()
    x, _ = mf.mustafar_paged_gather(cache, 16)
    got = x[0, 0, 3].float().cpu()
    want = row.bfloat16().float().clamp(-65504, 65504).half().float()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())


# ---- attention ---------------------------------------------------------------------------------
def attend(dtype, H, G, d, P, cached, new, window=0, sinks=0, scale=0.0, n_splits=0, seed=0, layout="heads", packed=False,
           junk=None, k_scale=1.0, **hints):
    lens = [a + b for a, b in zip(cached, new)]
    announce(f"attend {dtype} H={H} G={G} d={d} P={P} cached={cached} new={new} window={window} sinks={sinks} "
             f"splits={n_splits} layout={layout} packed={packed}")
    cache, ks, vs = fill(len(new), H, d, P, lens, dtype, seed=seed, layout=layout, junk=junk, k_scale=k_scale)
    g = torch.Generator().manual_seed(seed + 1)
    n_q = sum(new)
    x = torch.randn(n_q, H * G + (2 * H if packed else 0), d, generator=g).to(dtype).cuda()
    q = x[:, :H * G]
    out = torch.full((n_q, H * G + (1 if packed else 0), d), 9.0, dtype=dtype, device="cuda")[:, :H * G]
    got = mf.mustafar_paged_attn(q, cache, starts(new), window=window, sinks=sinks, scale=scale, n_splits=n_splits, out=out,
                                 **hints)
    torch.cuda.synchronize()
    worst = check(got, q, ks, vs, new, lens, dtype, window, sinks, scale if scale > 0 else None, label="attend")
    announce(f"  2-norm of the error: {worst:.2f} half steps of the type")
    return got, q, cache, ks, vs


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(2, 1), (1, 2), (2, 4), (1, 8), (1, 5), (1, 64)])
def test_single_tokens(dtype, d, H, G):
    attend(dtype, H, G, d, 16, [0, 1, 15, 63, 64, 200, 777], [1] * 7, seed=d + G)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(2, 1), (1, 3), (1, 8)])
@pytest.mark.parametrize("P", [16, 64, 256])
def test_chunks_of_prompts(dtype, d, H, G, P):
    attend(dtype, H, G, d, P, [0, 100, 0, 7, 63], [130, 65, 1, 33, 200], seed=d + G + P)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 4), (100, 0), (33, 70), (1000, 100)])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [70, 1, 0, 300]])
def test_windows_and_sinks(dtype, window, sinks, new):
    attend(dtype, 2, 2, 128, 32, [5, 400, 90, 130], new, window=window, sinks=sinks, seed=window)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40])
@pytest.mark.parametrize("sinks", [0, 2 ** 31 - 1])
@pytest.mark.parametrize("new", [[3, 2], [40, 100]])
def test_a_window_longer_than_anything(window, sinks, new):
    """Also for rows before a request's first token, whose window begins under -2^31."""
    cache, ks, vs = fill(2, 2, 128, 16, [2, 70], torch.float16, seed=30)
    q = torch.randn(sum(new), 4, 128, device="cuda").half()
    got = mf.mustafar_paged_attn(q, cache, starts(new), window=window, sinks=sinks)
    check(got, q, ks, vs, new, [2, 70], torch.float16, window, sinks, label="long window")


@pytest.mark.parametrize("dtype,d,n_splits", [(torch.float16, 64, 0), (torch.bfloat16, 64, 20), (torch.float16, 128, 3),
                                              (torch.bfloat16, 128, 20), (torch.float16, 256, 5), (torch.bfloat16, 256, 70)])
@pytest.mark.parametrize("B", [20, 65, 130])
def test_many_requests_of_single_tokens_and_a_few_chunks(dtype, d, n_splits, B):
    """Requests of few rows and of many side by side, every way of joining their ranges."""
    rng = random.Random(B + n_splits)
    cached = [rng.choice([0, 1, 30, 64, 200]) for _ in range(B)]
    new = [1] * B
    for b, n in ((0, 0), (3, 40), (B - 2, 70), (B - 1, 5)):
        new[b] = n
    attend(dtype, 2, 4, d, 16, cached, new, n_splits=n_splits, seed=B)
    attend(dtype, 2, 4, d, 16, cached, [min(n, 1) for n in new], n_splits=n_splits, seed=B)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_splits", [9, 63, 65, 100, 129, 700])
def test_more_ranges_than_a_wave_has_lanes(dtype, d, n_splits):
    """Few rows and many (a stream a row and a workgroup a row join them)."""
    attend(dtype, 1, 2, d, 64, [9000, 40], [1, 1], n_splits=n_splits, seed=n_splits)
    attend(dtype, 1, 4, d, 64, [5000, 40], [150, 1], n_splits=n_splits, seed=n_splits)


def test_as_many_requests_as_there_can_be():
    B = 4096
    rng = random.Random(1)
    lens = [rng.choice([0, 1, 2, 5, 17]) for _ in range(B)]
    new = [min(n, 1) for n in lens]
    new[1], lens[1] = 33, 40
    cache, ks, vs = fill(B, 1, 64, 16, lens, torch.float16, seed=31)
    q = torch.randn(sum(new), 1, 64, device="cuda").half()
    got = mf.mustafar_paged_attn(q, cache, starts(new), max_q=33)
    check(got, q, ks, vs, new, lens, torch.float16, label="4096")


@pytest.mark.parametrize("n_splits", [0, 5, 12, 70])
@pytest.mark.parametrize("new", [[1, 1, 1], [90, 1, 3], [40, 70, 33]])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_a_workspace_held_takes_no_part(d, new, n_splits):
    """A workspace of NaN: ranges without tokens, requests shorter than there are ranges, rows that see nothing."""
    cached = [3000, 2, 500]
    lens = [a + b for a, b in zip(cached, new)]
    cache, ks, vs = fill(3, 2, d, 16, lens, torch.float16, seed=60)
    cache.state[1] = 1              # fewer tokens than rows, where there is more than one
    lens[1], ks[1], vs[1] = 1, ks[1][:, :1], vs[1][:, :1]
    q = torch.randn(sum(new), 8, d, device="cuda").half()
    need = mf.mustafar_paged_attn_workspace_bytes(cache, 8, sum(new), max(new), 4000, n_splits)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    got = mf.mustafar_paged_attn(q, cache, starts(new), max_q=max(new), max_tokens=4000, n_splits=n_splits, ws=ws)
    check(got, q, ks, vs, new, lens, torch.float16, label="workspace of NaN")


def test_a_workspace_that_two_captured_calls_share():
    """Two graphs of calls of different sizes with one workspace, replayed in turns with eager calls between them."""
    dtype, made = torch.bfloat16, []
    for i, (cached, new) in enumerate((([3000, 40], [1, 1]), ([900, 100], [60, 1]))):
        lens = [a + b for a, b in zip(cached, new)]
        cache, ks, vs = fill(2, 2, 128, 16, lens, dtype, seed=40 + i)
        made.append((cache, ks, vs, lens, new, torch.randn(sum(new), 8, 128, device="cuda").to(dtype), starts(new)))
    need = max(mf.mustafar_paged_attn_workspace_bytes(m[0], 8, sum(m[4]), max(m[4]), max(m[3])) for m in made)
    assert need > 0
    ws, graphs, outs = torch.empty(need, dtype=torch.uint8, device="cuda"), [], []

    def call(m, out):
        mf.mustafar_paged_attn(m[5], m[0], m[6], max_q=max(m[4]), max_tokens=max(m[3]), out=out, ws=ws)
    for m in made:
        out = torch.zeros_like(m[5])
        call(m, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(m, out)
        graphs.append(graph)
        outs.append(out)
    for i in (0, 1, 1, 0, 0, 1):
        outs[i].fill_(9.0)
        graphs[i].replay()
        torch.cuda.synchronize()
        m = made[i]
        check(outs[i], m[5], m[1], m[2], m[4], m[3], dtype, label=f"graph {i}")
        again = torch.empty_like(m[5])
        call(m, again)
        assert torch.equal(again, outs[i])       # every call's sums are in one order


@pytest.mark.parametrize("n_splits", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("new,window,sinks", [([1, 1, 1], 0, 0), ([40, 1, 200], 0, 0), ([40, 1, 200], 130, 65)])
def test_splits(n_splits, new, window, sinks):
    attend(torch.bfloat16, 2, 4, 128, 16, [900, 3, 300], new, window=window, sinks=sinks, n_splits=n_splits, seed=n_splits)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [50, 150]])
def test_layouts_and_packed_rows(dtype, new):
    attend(dtype, 2, 4, 128, 32, [100, 300], new, layout="tokens", packed=True, seed=3)


def test_scale():
    attend(torch.float16, 2, 2, 64, 16, [100, 30], [1, 40], scale=0.03, seed=5)


def test_rows_without_tokens_and_rows_behind_the_last():
    """A request without new tokens, one that holds fewer tokens than it has rows, one that holds none; a
    padded batch."""
    for dtype in DTYPES:
        cache, ks, vs = fill(5, 2, 128, 16, [40, 0, 3, 70, 20], dtype, seed=1)
        new = [2, 3, 5, 0, 20]
        q = torch.randn(40, 8, 128, device="cuda").to(dtype)
        out = torch.full_like(q, 3.0)
        mf.mustafar_paged_attn(q, cache, starts(new), out=out)
        check(out, q, ks, vs, new, [40, 0, 3, 70, 20], dtype, label="empty")
        assert bool((out[30:] == 3).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new", [[1, 1, 1], [90, 1, 17]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_what_no_row_sees_takes_no_part(dtype, junk, new, window, sinks):
    """Pages' unwritten rows hold NaN or infinities; table entries of pages out of every row's sight are bad."""
    cached = [200, 17, 64]
    lens = [a + b for a, b in zip(cached, new)]
    cache, ks, vs = fill(3, 2, 128, 16, lens, dtype, seed=2, junk=junk)
    if window:
        for b, (n, L) in enumerate(zip(new, lens)):
            for i in range((L + 15) // 16):
                if i * 16 >= sinks and i * 16 + 15 <= L - n - window:
                    cache.table[b, i] = random.Random(i).choice([-1, 1 << 30])
    q = torch.randn(sum(new), 8, 128, device="cuda").to(dtype)
    got = mf.mustafar_paged_attn(q, cache, starts(new), window=window, sinks=sinks)
    check(got, q, ks, vs, new, lens, dtype, window, sinks, label="junk")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 2)])
@pytest.mark.parametrize("G", [1, 4])
def test_infinities_and_nan_of_tokens_that_some_rows_see(dtype, bad, window, sinks, G):
    """A value (and in another request a key) that is not finite reaches the rows that see it and no other."""
    cached, new = [70, 150, 10], [60, 100, 1]
    lens = [a + b for a, b in zip(cached, new)]
    cache, ks, vs = fill(3, 1, 128, 16, lens, dtype, seed=4)
    for b, j, which in ((0, 100, "v"), (1, 200, "k"), (2, 3, "v")):
        page, at = int(cache.table[b, j // 16]), j % 16
        (cache.v if which == "v" else cache.k)[page, 0, at, 5] = bad
        (vs if which == "v" else ks)[b][0, j, 5] = bad
    q = torch.randn(sum(new), G, 128, device="cuda").to(dtype)
    got = mf.mustafar_paged_attn(q, cache, starts(new), window=window, sinks=sinks)
    check(got, q, ks, vs, new, lens, dtype, window, sinks, label="not finite")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [70, 33]])
@pytest.mark.parametrize("k_scale", [30.0, 1000.0])
def test_large_scores(dtype, new, k_scale):
    """Scores of hundreds and of tens of thousands: one token takes nearly all the weight."""
    attend(dtype, 1, 4, 128, 16, [300, 50], new, k_scale=k_scale, seed=6)


def test_all_scores_very_low():
    """Every score far under zero: the softmax's shift follows them down."""
    for dtype in DTYPES:
        cache, ks, vs = fill(1, 1, 64, 16, [200], dtype, seed=8)
        cache.k.copy_(-cache.k.abs() * 20)
        ks = [-ks[0].abs() * 20]
        for n in (1, 77):
            q = torch.rand(n, 4, 64, device="cuda").to(dtype) * 8 + 1
            got = mf.mustafar_paged_attn(q, cache, starts([n]))
            check(got, q, ks, vs, [n], [200], dtype, label="low")


@pytest.mark.parametrize("late", [False, True])
def test_one_token_far_above_the_others(late):
    """A token 20 log2 units above 60000 others: the small weights' sum counts."""
    L, d = 60001, 64
    for dtype in DTYPES:
        cache, ks, vs = fill(1, 1, d, 64, [L], dtype, seed=9, k_scale=0.05)
        vs[0] += 1
        q = torch.ones(1, 2, d).to(dtype).cuda()
        j = L - 3 if late else 2
        ks[0][0, j] = 14 * 0.6931 / 8
        cache2, _, _ = cache, None, None
        page, at = int(cache2.table[0, j // 64]), j % 64
        cache2.k[page, 0, at] = ks[0][0, j].cuda()
        cache2.v += 1
        vs = [v.cuda() for v in vs]
        for i in range((L + 63) // 64):
            m = min(64, L - 64 * i)
            cache2.v[cache2.table[0, i].long(), :, :m] = vs[0][:, 64 * i:64 * i + m]
        got = mf.mustafar_paged_attn(q, cache2, starts([1]))
        check(got, q, ks, vs, [1], [L], dtype, label="peak")


@pytest.mark.parametrize("dtype,new", [(torch.bfloat16, [1, 1, 1]), (torch.float16, [1, 300, 64])])
def test_long_requests(dtype, new):
    attend(dtype, 2, 4, 128, 64, [20000, 9000, 131], new, seed=10)


@pytest.mark.parametrize("new", [[1, 1], [64, 5]])
def test_hints_only_choose(new):
    """Bounds that are too small or too large give the same result within the types' rounding."""
    for max_q, max_tokens in ((1, 1), (1, 5000), (64, 700), (1000, 100000), (0, 0)):
        attend(torch.float16, 2, 4, 128, 16, [500, 600], new, max_q=max_q, max_tokens=max_tokens, seed=11)


def test_a_length_beyond_the_table_is_read_as_the_tables():
    cache, ks, vs = fill(1, 1, 64, 16, [64], torch.float16, seed=12, max_pages=4)
    cache.state[0] = 70        # 64 tokens fit
    q = torch.randn(1, 1, 64, device="cuda").half()
    got = mf.mustafar_paged_attn(q, cache, starts([1]))
    check(got, q, ks, vs, [1], [64], torch.float16, label="beyond")


def test_pools_of_more_than_two_to_the_31_elements():
    """Pages whose offsets pass 32 bits, in bytes and in elements."""
    H, d, P = 8, 256, 1024
    n_pages = (1 << 31) // (H * d * P) + 40
    pool = [torch.empty((n_pages, H, P, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = mf.PagedCache(2, H, d, n_pages, P, max_pages=4, k=pool[0], v=pool[1])
    new = [1500, 1030]
    cu, slots = mf.mustafar_paged_plan(cache, ints(new), sum(new))
    cache.table.copy_(n_pages - 1 - cache.table)    # the last pages of the pool
    slots = (n_pages - 1 - slots // P) * P + slots % P
    assert int(cache.table[0, 0]) == n_pages - 1 and (n_pages - 4) * H * P * d > 1 << 31
    x = torch.randn(sum(new), 3 * H, d, device="cuda").bfloat16()
    q, k, v = x[:, :H], x[:, H:2 * H], x[:, 2 * H:]
    mf.mustafar_paged_write(cache, k, v, slots.int())
    got = mf.mustafar_paged_attn(q[-1100:], cache, starts([70, 1030]))
    ks = [k[:1500].transpose(0, 1), k[1500:].transpose(0, 1)]
    vs = [v[:1500].transpose(0, 1), v[1500:].transpose(0, 1)]
    check(got, q[-1100:], ks, vs, [70, 1030], new, torch.bfloat16, label="far pages")
    x_k, _ = mf.mustafar_paged_gather(cache, 1500)
    assert torch.equal(x_k[0], ks[0].float().half())


# ---- together ----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_serving_loop_from_prompts_to_compressed_caches(dtype):
    """Prompts in chunks through plan, write and attention, each chunk against float64; then the pages become
    compressed caches and a window whose decode attention is the oracle's."""
    B, H, G, d, P, W = 3, 2, 4, 128, 16, 32
    lens = [150, 77, 201]
    g = torch.Generator().manual_seed(13)
    k = [torch.randn(n + 1, H, d, generator=g).to(dtype).cuda() for n in lens]
    v = [torch.randn(n + 1, H, d, generator=g).to(dtype).cuda() for n in lens]
    cache = mf.PagedCache(B, H, d, 40, P, max_pages=20, dtype=dtype)
    done = [0] * B
    for chunk in (64, 50, 1, 100):
        new = [min(chunk, n - m) for n, m in zip(lens, done)]
        n = sum(new) + 5                                    # a padded step
        cu, slots = mf.mustafar_paged_plan(cache, ints(new), n)
        rows = [x[m:m + a] for x, m, a in zip(k, done, new)], [x[m:m + a] for x, m, a in zip(v, done, new)]
        pad = torch.full((5, H, d), float("nan"), dtype=dtype, device="cuda")
        mf.mustafar_paged_write(cache, torch.cat(rows[0] + [pad]), torch.cat(rows[1] + [pad]), slots)
        q = torch.randn(n, H * G, d, device="cuda").to(dtype)
        out = mf.mustafar_paged_attn(q, cache, cu, out=torch.full_like(q, 5.0))
        done = [m + a for m, a in zip(done, new)]
        check(out, q, [x[:m].transpose(0, 1) for x, m in zip(k, done)], [x[:m].transpose(0, 1) for x, m in zip(v, done)], new,
              done, dtype, label=f"chunk {chunk}")
        assert bool((out[-5:] == 5).all())
    assert done == lens
    x_k, x_v = mf.mustafar_paged_gather(cache, max(lens))
    Kc, Vc, win = mf.CompressedCache(B, H, d, 0.5, 256), mf.CompressedCache(B, H, d, 0.7, 256), mf.DenseWindow(B, H, d, W)
    mf.mustafar_window_prefill(win, Kc, Vc, x_k, x_v, lens)
    q = torch.randn(B, H * G, d, device="cuda").half()
    out = mf.mustafar_window_decode_attn(q, Kc, Vc, win).cpu().numpy()
    for b, n in enumerate(lens):
        kb, vb = (np.ascontiguousarray(x[b][:n].transpose(0, 1).float().half().cpu().numpy())[None] for x in (k, v))
        want = oracle.sparse_decode_attention(q[b:b + 1].cpu().numpy(), oracle.compress(np.ascontiguousarray(kb[:, :, :n - W]), 0.5),
                                              oracle.compress(np.ascontiguousarray(vb[:, :, :n - W]), 0.7),
                                              np.ascontiguousarray(kb[:, :, n - W:]), np.ascontiguousarray(vb[:, :, n - W:]))
        assert attn_error(out[b:b + 1], want) <= ATTN_TOL
    mf.mustafar_paged_plan(cache, ints([0] * B), 0, keep=ints([0] * B))        # the requests' pages are free again
    assert cache.state.tolist() == [0, 0, 0, 40, 0] and sorted(cache.free.tolist()) == list(range(40))


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_captured_step_replays(dtype):
    """Plan, write and attention of a step in one graph, replayed with eager work between the replays: every
    replay advances the state and gives what eager calls on a second cache give."""
    B, H, G, d, P = 3, 2, 4, 128, 16
    lens = [100, 31, 500]
    caches = [fill(B, H, d, P, lens, dtype, seed=14, spare=60, max_pages=64)[0] for _ in range(2)]
    # the pages behind the tables' are the same in both
    new = ints([1, 40, 9])
    n = 60
    rows = [torch.randn(n, (G + 2) * H, d, device="cuda").to(dtype) for _ in range(4)]
    x = rows[0].clone()
    cu, slots, status = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), ints([0])
    out = torch.zeros(n, H * G, d, dtype=dtype, device="cuda")
    need = mf.mustafar_paged_attn_workspace_bytes(caches[0], H * G, n, 40, 1000)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def step(cache, x, cu, slots, status, out):
        mf.mustafar_paged_plan(cache, new, n, cu=cu, slots=slots, status=status)
        mf.mustafar_paged_write(cache, x[:, H * G:H * (G + 1)], x[:, H * (G + 1):], slots)
        return mf.mustafar_paged_attn(x[:, :H * G], cache, cu, max_q=40, max_tokens=1000, out=out, ws=ws)

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(caches[0], x, cu, slots, status, out)
    for r in range(4):
        x.copy_(rows[r])
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = step(caches[1], rows[r], cu.clone(), slots.clone(), status.clone(), torch.zeros_like(out))
        torch.cuda.synchronize()
        assert status.tolist() == [0] and caches[0].lens.tolist() == [a + (r + 1) * b for a, b in zip(lens, [1, 40, 9])]
        assert torch.equal(caches[0].state, caches[1].state) and torch.equal(got, want), r


def test_other_streams():
    """Calls on a stream that is not the current one, two streams at once."""
    dtype, results = torch.float16, []
    made = [fill(2, 2, 128, 16, [700, 300], dtype, seed=s) for s in (20, 21)]
    qs = [torch.randn(130, 8, 128, device="cuda").to(dtype) for _ in range(2)]
    cu = starts([100, 30])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        outs = [mf.mustafar_paged_attn(q, m[0], cu, stream=s) for q, m, s in zip(qs, made, streams)]
        torch.cuda.synchronize()
        results.append(outs)
    for outs in results:
        for out, q, m in zip(outs, qs, made):
            check(out, q, m[1], m[2], [100, 30], [700, 300], dtype, label="streams")


def test_the_binding_refuses_what_does_not_fit():
    """Shapes, types, strides and devices are checked before anything is launched."""
    cache, _, _ = fill(2, 2, 64, 16, [20, 30], torch.float16, seed=50)
    state = cache.state.clone()
    x = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    q, cu, slots = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda"), starts([1, 1]), ints([0, 1, 2])
    plan = lambda **kw: mf.mustafar_paged_plan(**{**dict(cache=cache, new_len=ints([1, 1]), n_slots=2), **kw})  # noqa: E731
    write = lambda **kw: mf.mustafar_paged_write(**{**dict(cache=cache, k_new=x, v_new=x, slots=slots), **kw})  # noqa: E731
    attn = lambda **kw: mf.mustafar_paged_attn(**{**dict(q=q, cache=cache, cu=cu), **kw})  # noqa: E731
    gather = lambda **kw: mf.mustafar_paged_gather(**{**dict(cache=cache, n_max=4), **kw})  # noqa: E731
    bad = [(plan, dict(new_len=ints([1]))), (plan, dict(new_len=ints([1, 1]).cpu())), (plan, dict(new_len=ints([1, 1]).long())),
           (plan, dict(keep=ints([1, 1, 1]))), (plan, dict(state_out=ints([0, 0]))), (plan, dict(slots=ints([0]))),
           (write, dict(k_new=x.float())), (write, dict(v_new=x[:2])), (write, dict(k_new=x.cpu())), (write, dict(k_new=x[:, :1])),
           (write, dict(k_new=x.transpose(0, 1).contiguous().transpose(0, 1))), (write, dict(slots=slots[:2])),
           (write, dict(slots=slots.long())), (attn, dict(q=q.bfloat16())), (attn, dict(q=q[0])), (attn, dict(q=q[..., :32])),
           (attn, dict(q=q.cpu())), (attn, dict(cu=cu[:2])), (attn, dict(cu=cu.long())), (attn, dict(out=q[:1])),
           (attn, dict(out=q.float())), (attn, dict(out=q.cpu())), (attn, dict(ws=torch.zeros(1 << 20))),
           (gather, dict(first=ints([0]))), (gather, dict(x_k=x)), (gather, dict(x_k=torch.zeros(2, 2, 4, 64, device="cuda")))]
    for call, kw in bad:
        with pytest.raises(ValueError):
            call(**kw)
    for call, kw in ((attn, dict(q=torch.zeros(2, 3, 64, dtype=torch.float16, device="cuda"))), (attn, dict(window=-1)),
                     (attn, dict(n_splits=4, ws=torch.zeros(16, dtype=torch.uint8, device="cuda"))),
                     (attn, dict(q=torch.zeros(2, 130, 64, dtype=torch.float16, device="cuda"))), (plan, dict(n_slots=-1, slots=ints([])))):
        with pytest.raises((mf.MustafarError, ValueError)):
            call(**kw)
    assert torch.equal(cache.state, state)
    for call, kw in ((attn, dict(q=q[:0], cu=starts([0, 0]))), (write, dict(k_new=x[:0], v_new=x[:0], slots=slots[:0])),
                     (plan, dict(new_len=ints([0, 0]), n_slots=0)), (gather, dict(n_max=0))):
        call(**kw)                                                                     # nothing to do
    torch.cuda.synchronize()
    assert torch.equal(cache.state, state)
