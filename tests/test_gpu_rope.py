"""Rotary positions on the GPU against float64."""
import math

import pytest
import torch

import paper_2505_22913_amd as mf
from oracle import paged8 as oracle8
from tests.gpu_common import announce
from tests.paged_common import starts

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def close(got, x, positions, rates, rot, layout, magnitude=1.0, inverse=False):
    """Every element within its rounding to the type (half a step of it; 2^-25 where fp16's steps stop falling) and what
    fp32 makes: cosine and sine are off by at most 4 steps of 2^-24 (the reduced angle's rounding, times 2 pi, and theirs; the
    magnitude's product one more), each product and their sum by one."""
    want, mag = oracle8.rotate(x.cpu(), positions, rates, rot, layout, magnitude, inverse)
    u = torch.finfo(x.dtype).eps / 2
    err = (got.cpu().double() - want).abs()
    assert bool((err <= u * want.abs() + 8 * 2.0 ** -24 * mag * (1 + u) + 2.0 ** -25 * (mag > 0)).all()), float((err - u * want.abs()).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (256, 256), (512, 512), (128, 64), (80, 32), (80, 20), (96, 96), (8, 2), (8, 8),
                                   (128, 126), (64, 6), (512, 500), (24, 16)])
@pytest.mark.parametrize("Hq,H", [(1, 0), (5, 2)])
def test_layouts_parts_and_sizes(dtype, layout, d, rot, Hq, H):
    announce(f"rope {dtype} {layout} d={d} rot={rot} Hq={Hq} H={H}")
    rope = mf.Rope(rot, 10000.0, layout, magnitude=0.75)
    rates = oracle8.rates(rot, 10000.0)
    for n in (1, 3, 9):
        g = torch.Generator().manual_seed(n + d + rot)
        x = torch.randn(n, Hq + H, d, generator=g).to(dtype)
        positions = torch.randint(-70000, 70000, (n,), generator=g).int()
        on, pos = x.cuda(), positions.cuda()
        q, k = on[:, :Hq], on[:, Hq:] if H else None
        for inverse in (False, True):
            out_q, out_k = mf.mustafar_rope(rope, q, k, positions=pos, inverse=inverse)
            assert torch.equal(on.cpu(), x)
            got = out_q if k is None else torch.cat([out_q, out_k], 1)
            close(got, x, positions, rates, rot, layout, 0.75, inverse)
            assert torch.equal(got[..., rot:].cpu(), x[..., rot:])
            # in place, in the packed rows, and with one of the two in place
            packed = torch.cat([on, torch.full((n, 1, d), 9.0, dtype=dtype, device="cuda")], 1)
            pq, pk = packed[:, :Hq], packed[:, Hq:Hq + H] if H else None
            mf.mustafar_rope(rope, pq, pk, positions=pos, inverse=inverse, out_q=pq, out_k=pk)
            assert torch.equal(packed[:, :Hq + H], got) and bool((packed[:, -1] == 9).all())
            if H:
                again = on.clone()
                _, other = mf.mustafar_rope(rope, again[:, :Hq], again[:, Hq:], positions=pos, inverse=inverse, out_q=again[:, :Hq])
                assert torch.equal(again[:, :Hq], out_q) and torch.equal(other, out_k) and torch.equal(again[:, Hq:], on[:, Hq:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot,Hq,H", [(512, 510, 20, 3), (512, 18, 40, 8), (80, 20, 33, 31), (256, 254, 64, 8), (16, 2, 1, 1)])
def test_many_heads_whose_pairs_lie_in_no_pieces(layout, d, rot, Hq, H):
    x = torch.randn(6, Hq + H, d, generator=torch.Generator().manual_seed(d + rot)).bfloat16()
    positions = torch.tensor([0, 5, -3, 70000, 1, 2], dtype=torch.int32)
    on = x.cuda()
    q, k = mf.mustafar_rope(mf.Rope(rot, layout=layout), on[:, :Hq], on[:, Hq:], positions=positions.cuda())
    close(torch.cat([q, k], 1), x, positions, oracle8.rates(rot, 10000.0), rot, layout)
    assert torch.equal(torch.cat([q, k], 1)[..., rot:], on[..., rot:])


@pytest.mark.parametrize("layout,rot", [("half", 128), ("interleaved", 64), ("half", 36)])
def test_rows_that_the_caches_do_not_hold(layout, rot):
    """Inputs and outputs of 205 MB."""
    n, Hq, H, d = 10000, 32, 8, 128
    x = torch.randn(n, Hq + H, d, device="cuda").half()
    pos = torch.arange(n, device="cuda").int() * 3
    q, k = mf.mustafar_rope(mf.Rope(rot, layout=layout), x[:, :Hq], x[:, Hq:], positions=pos)
    rows = list(range(0, n, 397)) + [n - 1]
    close(torch.cat([q, k], 1)[rows], x[rows], pos[rows].cpu(), oracle8.rates(rot, 10000.0), rot, layout)
    packed = x.clone()
    mf.mustafar_rope(mf.Rope(rot, layout=layout), packed[:, :Hq], packed[:, Hq:], positions=pos, out_q=packed[:, :Hq], out_k=packed[:, Hq:])
    assert torch.equal(packed, torch.cat([q, k], 1))


@pytest.mark.parametrize("scaling,kw", [("linear", dict(factor=8.0)), ("base", dict(factor=4.0)),
                                        ("turns", dict(factor=8.0, original_len=8192, low_turns=1.0, high_turns=4.0))])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rates_for_long_contexts_at_far_positions(dtype, scaling, kw):
    """Positions up to 2^31: the angle is as exact as at 0."""
    d = 128
    rope = mf.Rope(d, 500000.0, "half", scaling, **kw)
    rates = oracle8.rates(d, 500000.0, scaling, kw["factor"], kw.get("original_len", 0), kw.get("low_turns", 1), kw.get("high_turns", 32))
    assert torch.allclose(rope.rates.cpu(), torch.tensor(rates, dtype=torch.float64), rtol=1e-14, atol=0)
    rates = rope.rates.tolist()         # (the same numbers: their last bit is 2^-21 radians at these positions)
    positions = torch.tensor([0, 1, 131071, 1048576, 10 ** 8 + 7], dtype=torch.int32)
    x = torch.randn(5, 3, d, generator=torch.Generator().manual_seed(3)).to(dtype)
    out, _ = mf.mustafar_rope(rope, x.cuda(), positions=positions.cuda())
    close(out, x, positions, rates, d, "half")
    # the last positions that 32 bits hold: p r / (2 pi) is rounded twice in 53 bits, 2^31 turns' fraction to 2^-21 of a turn
    positions = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 5, 6], dtype=torch.int32)
    out, _ = mf.mustafar_rope(rope, x.cuda(), positions=positions.cuda())
    want, mag = oracle8.rotate(x, positions, rates, d, "half")
    u = torch.finfo(dtype).eps / 2
    assert bool(((out.cpu().double() - want).abs() <= u * want.abs() + mag * (8 * 2.0 ** -24 + 2 * math.pi * 2.0 ** -20) + 2.0 ** -25).all())


@pytest.mark.parametrize("B", [1, 3, 64, 65, 300])
@pytest.mark.parametrize("by", ["dense", "codes"])
def test_positions_of_a_planned_step(B, by):
    """Ragged requests, some without tokens, a padded step, a refused one."""
    d, rot, g = 64, 64, torch.Generator().manual_seed(B)
    kind = mf.PagedCache if by == "dense" else mf.PagedCache8
    cache = kind(B, 1, 64, 4 * B + 40, 16, max_pages=30)
    rope, rates = mf.Rope(rot), oracle8.rates(rot, 10000.0)
    lens = [0] * B
    for i in range(3):
        new = torch.randint(0, 4, (B,), generator=g).tolist()
        new[B // 2] = 17
        n = sum(new) + 6
        cu, _ = mf.mustafar_paged_plan(cache, ints(new), n)
        assert cache.status.tolist() == [0]
        x = torch.randn(n, 3, d, generator=g).half()
        on = x.cuda()
        out_q, out_k = mf.mustafar_rope(rope, on[:, :2], on[:, 2:], cache=cache, cu=cu, out_q=torch.full((n, 2, d), 5.0, dtype=torch.float16, device="cuda"))
        pos = torch.cat([torch.arange(m, m + a) for m, a in zip(lens, new)]).int()
        close(torch.cat([out_q, out_k], 1)[:n - 6], x[:n - 6], pos, rates, rot, "half")
        assert bool((out_q[n - 6:] == 5).all()) and bool((out_k[n - 6:] == 0).all())
        lens = [m + a for m, a in zip(lens, new)]
    cu, _ = mf.mustafar_paged_plan(cache, ints([4000] * B), 10)
    assert cache.status.tolist() != [0]
    mf.mustafar_rope(rope, on[:, :2], cache=cache, cu=cu, out_q=on[:, :2])
    assert torch.equal(on.cpu(), x)


def test_rows_of_a_request_that_holds_fewer_tokens_turn_back_and_lengths_end_with_the_table():
    cache = mf.PagedCache(2, 1, 64, 4, 16, max_pages=2)
    cache.state.copy_(ints([3, 40, 0, 0]))             # 32 tokens fit
    rope, rates = mf.Rope(64, layout="interleaved"), oracle8.rates(64, 10000.0)
    x = torch.randn(7, 1, 64, generator=torch.Generator().manual_seed(1)).half()
    out, _ = mf.mustafar_rope(rope, x.cuda(), cache=cache, cu=starts([5, 2]))
    close(out, x, torch.tensor([-2, -1, 0, 1, 2, 30, 31]), rates, 64, "interleaved")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [64, 22])
def test_the_gradient_is_the_rotation_back(layout, rot):
    """<w, R x>'s gradient in x is R^T w: against differences of the formula in float64, and against autograd of it."""
    d, n = 64, 4
    g = torch.Generator().manual_seed(rot)
    rates, positions = oracle8.rates(rot, 10000.0), torch.tensor([0, 7, 1000, 123456], dtype=torch.int32)
    x = torch.randn(n, 2, d, generator=g).half().double()
    w = torch.randn(n, 2, d, generator=g).half()
    rope = mf.Rope(rot, layout=layout, magnitude=1.25)
    got, _ = mf.mustafar_rope(rope, w.cuda(), positions=positions.cuda(), inverse=True)
    close(got, w, positions, rates, rot, layout, 1.25, True)
    tol = 2.0 ** -11 * 1.25 * 4 + 1e-6       # half a step of values under 8, and what the differences leave
    for t, h, c in ((0, 0, 0), (1, 1, rot - 1), (2, 0, rot // 2), (3, 1, 5), (3, 0, 63)):
        step = torch.zeros_like(x)
        step[t, h, c] = 1e-3
        loss = [(oracle8.rotate(x + s * step, positions, rates, rot, layout, 1.25)[0] * w.double()).sum() for s in (1, -1)]
        assert abs(float(loss[0] - loss[1]) / 2e-3 - float(got[t, h, c])) <= tol
    xa = x.clone().requires_grad_()
    a = xa[..., :rot // 2] if layout == "half" else xa[..., 0:rot:2]
    b = xa[..., rot // 2:rot] if layout == "half" else xa[..., 1:rot:2]
    angle = positions.double()[:, None, None] * torch.tensor(rates, dtype=torch.float64)
    ya, yb = (a * angle.cos() - b * angle.sin()) * 1.25, (a * angle.sin() + b * angle.cos()) * 1.25
    wa = w[..., :rot // 2] if layout == "half" else w[..., 0:rot:2]
    wb = w[..., rot // 2:rot] if layout == "half" else w[..., 1:rot:2]
    ((ya * wa).sum() + (yb * wb).sum() + (xa[..., rot:] * w[..., rot:]).sum()).backward()
    assert bool(((got.cpu().double() - xa.grad).abs() <= 2.0 ** -11 * xa.grad.abs() + 1e-5).all())


def test_infinities_and_nan_stay_in_their_pair():
    for layout, rot in (("half", 64), ("interleaved", 64), ("half", 20), ("interleaved", 20)):
        x = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(2)).half()
        bad = x.clone()
        bad[0, 1, 3], bad[1, 0, 9] = float("inf"), float("nan")
        rope, positions = mf.Rope(rot, layout=layout), ints([5, 9])
        got, _ = mf.mustafar_rope(rope, bad.cuda(), positions=positions)
        want, _ = mf.mustafar_rope(rope, x.cuda(), positions=positions)
        for t, h, c in ((0, 1, 3), (1, 0, 9)):
            other = (c + rot // 2 if c < rot // 2 else c - rot // 2) if layout == "half" else c ^ 1
            for i in (c, other):
                assert not bool(torch.isfinite(got[t, h, i]))
                got[t, h, i] = want[t, h, i]
        assert torch.equal(got, want)


def test_many_rows_and_heads_on_other_streams_and_in_a_graph():
    n, Hq, H, d = 5000, 32, 8, 128
    rope = mf.Rope(d, layout="interleaved")
    x = torch.randn(n, Hq + H, d, device="cuda").bfloat16()
    pos = torch.arange(n, device="cuda").int()
    want = mf.mustafar_rope(rope, x[:, :Hq], x[:, Hq:], positions=pos)
    rows = [0, 1, 77, 4095, 4999]
    close(want[0][rows], x[rows, :Hq], pos[rows].cpu(), oracle8.rates(d, 10000.0), d, "interleaved")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [mf.mustafar_rope(rope, x[:, :Hq], x[:, Hq:], positions=pos, stream=s) for s in streams]
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    q, k, graph = torch.zeros_like(want[0]), torch.zeros_like(want[1]), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mf.mustafar_rope(rope, x[:, :Hq], x[:, Hq:], positions=pos, out_q=q, out_k=k)
    for i in range(3):
        pos += 1
        graph.replay()
        torch.cuda.synchronize()
        again = mf.mustafar_rope(rope, x[:, :Hq], x[:, Hq:], positions=pos)
        assert torch.equal(q, again[0]) and torch.equal(k, again[1])


def test_the_binding_refuses_what_does_not_fit():
    rope = mf.Rope(64)
    x = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    pos, cache = ints([0, 1, 2]), mf.PagedCache(2, 2, 64, 8, 16)
    call = lambda **kw: mf.mustafar_rope(**{**dict(rope=rope, q=x, positions=pos), **kw})  # noqa: E731
    for kw in (dict(q=x.float()), dict(q=x[0]), dict(q=x.cpu()), dict(k=x[:2]), dict(k=x.bfloat16()), dict(k=x[..., :32]), dict(positions=None),
               dict(cache=cache, cu=starts([1, 2])), dict(positions=None, cache=cache), dict(positions=pos[:2]), dict(positions=pos.long()),
               dict(positions=pos.cpu()), dict(out_q=x[:2]), dict(out_q=x.float()), dict(out_k=x), dict(positions=None, cache=cache, cu=pos[:2]),
               dict(q=x.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            call(**kw)
    wide = torch.zeros(3, 5, 64, dtype=torch.float16, device="cuda")
    for kw in (dict(q=x[..., :32].contiguous()), dict(q=torch.zeros(3, 2, 76, dtype=torch.float16, device="cuda")),
               dict(q=torch.zeros(3 * 128 + 1, dtype=torch.float16, device="cuda")[1:].view(3, 2, 64)),
               dict(q=wide.view(-1)[:3 * 260].as_strided((3, 2, 64), (260 + 2, 64, 1), 0)),
               dict(q=torch.zeros(3, 1, 520, dtype=torch.float16, device="cuda"))):
        with pytest.raises(mf.MustafarError):
            call(**kw)
    for kw in (dict(rot=0), dict(rot=63), dict(rot=64, base=0.0), dict(rot=64, base=float("nan")), dict(rot=2, scaling="base", factor=2.0),
               dict(rot=64, scaling="linear", factor=0.0), dict(rot=64, scaling="turns", factor=2.0)):
        with pytest.raises(mf.MustafarError):
            mf.Rope(**kw)
    for kw in (dict(rot=64, layout="quarter"), dict(rot=64, scaling="other"), dict(rot=64, rates=torch.zeros(32, device="cuda")),
               dict(rot=64, rates=torch.zeros(31, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            mf.Rope(**kw)
    out, none = call(q=x[:0], positions=pos[:0])
    assert out.shape == (0, 2, 64) and none is None
