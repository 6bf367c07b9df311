"""The paged dense cache and what works on it, as cases that can be timed and compared.

A case is a dict of plain values; `kind` names the operator:

  plan    block tables, slots and sequence starts of a step, from the requests' lengths
          (`mustafar_paged_plan`)
  write   keys and values of new tokens into their slots (`mustafar_paged_write`)
  gather  requests' pages as the dense fp16 tensors that the compression takes
          (`mustafar_paged_gather`)
  attend  causal attention of every request's new tokens over its pages, with or without a
          sliding window and first tokens that stay visible (`mustafar_paged_attn`)

`own` selects the library's kernels; without it every operator is computed with elementary
torch operations in 32 bits. Sizes are those of the library's synthetic workloads (layers of 8 or
32 kv-heads, 1 to 8 query heads each, one sequence of 4K tokens to batches of 16K and 32K) and
of the steps of a serving loop.
"""
import math

import torch

own = False     # the library's kernels instead of the plain forms

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
PAIR_LIMIT = 1 << 42    # products of 64-bit pairs above which the exact answer takes too long


def listed():
    return [
        # A decode step of 64 running requests: one token each, a few of which open a page.
        dict(name="plan_decode_b64", kind="plan", B=64, P=64, cached=8192, new=1, replaced=0),
        # A step that admits and continues prompts on small pages; every eighth request is a new one
        # in the place of a finished one.
        dict(name="plan_prompts_b256_p16", kind="plan", B=256, P=16, cached=16384, new=512, replaced=8),
        # The keys and values of that decode step.
        dict(name="write_decode_b64", kind="write", n=64, H=8, d=128, P=64, dtype="fp16", packed=False),
        # A large prompt step, read out of the packed projection.
        dict(name="write_prompt_16k_bf16", kind="write", n=16384, H=8, d=128, P=16, dtype="bf16", packed=True),
        # One short prompt on its way to the compressed cache.
        dict(name="gather_b1_mha_1k", kind="gather", B=1, H=32, d=128, P=64, n=1000, first=0, dtype="fp16"),
        # A batch of long prompts of a bf16 model, rounded to the compressed caches' fp16.
        dict(name="gather_b8_gqa_16k_bf16", kind="gather", B=8, H=8, d=128, P=64, n=16384, first=0, dtype="bf16"),
        # One chat sequence of 4K tokens on a 32-head layer: the latency of a single call.
        dict(name="attend_decode_b1_mha_4k", kind="attend", B=1, Hq=32, H=32, d=128, P=64, cached=4095, new=1,
             ragged=False, window=0, sinks=0, dtype="fp16", packed=False),
        # A continuous batch of different lengths on a grouped-query layer with small pages.
        dict(name="attend_decode_b16_gqa4_16k_ragged_bf16", kind="attend", B=16, Hq=32, H=8, d=128, P=16,
             cached=16384, new=1, ragged=True, window=0, sinks=0, dtype="bf16", packed=False),
        # Long sequences of which each token sees the newest 1024 and four first ones.
        dict(name="attend_decode_b32_gqa8_d64_32k_window", kind="attend", B=32, Hq=64, H=8, d=64, P=32,
             cached=32768, new=1, ragged=False, window=1024, sinks=4, dtype="fp16", packed=False),
        # A chunk of a long prompt whose first 16K tokens are in the cache.
        dict(name="attend_chunk_512_of_16k_gqa4", kind="attend", B=1, Hq=32, H=8, d=128, P=64, cached=16384,
             new=512, ragged=False, window=0, sinks=0, dtype="fp16", packed=False),
        # Whole prompts on a 32-head layer: the largest amount of arithmetic.
        dict(name="attend_prompts_b4_mha_4k_bf16", kind="attend", B=4, Hq=32, H=32, d=128, P=64, cached=0,
             new=4096, ragged=False, window=0, sinks=0, dtype="bf16", packed=False),
        # A mixed step: prompts' chunks of very different lengths beside single tokens, with a window,
        # queries read out of the packed projection.
        dict(name="attend_mixed_b16_gqa4_window_bf16", kind="attend", B=16, Hq=32, H=8, d=128, P=32, cached=8192,
             new=1024, ragged=True, window=4096, sinks=4, dtype="bf16", packed=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "write", "gather"] + ["attend"] * 5)
    P, dtype = rng.choice([16, 32, 64, 64, 128, 256]), rng.choice(["fp16", "bf16"])
    d, H = rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 8, 8, 16, 32])
    if kind == "plan":
        return dict(kind=kind, B=_log_int(rng, 1, 256), P=P, cached=_log_int(rng, 1, 32768),
                    new=rng.choice([1, 1, _log_int(rng, 2, 512)]), replaced=rng.choice([0, 0, 3, 8]))
    if kind == "write":
        n = _log_int(rng, 1, min(16384, 16384 * 1024 // (H * d)))
        return dict(kind=kind, n=n, H=H, d=d, P=P, dtype=dtype, packed=rng.random() < 0.5)
    if kind == "gather":
        B = _log_int(rng, 1, 16)
        n = _log_int(rng, 1, max(1, min(32768, (1 << 27) // (B * H * d))))
        return dict(kind=kind, B=B, H=H, d=d, P=P, n=n, first=rng.choice([0, 0, rng.randint(1, 4096)]), dtype=dtype)
    G = rng.choice([1, 2, 3, 4, 4, 7, 8])
    B = _log_int(rng, 1, 32)
    most = (1 << 28) // (B * H * d)     # cached tokens per request: up to 1 GiB of 16-bit keys and values
    cached = _log_int(rng, 1, max(1, min(65536, most)))
    new = 1
    if rng.random() < 0.6:
        # the scores of a whole batch, and fewer products than the largest listed case
        heads = B * H * G
        new = min((1 << 28) // (heads * cached), math.isqrt((1 << 36) // (heads * d)), (1 << 28) // (heads * d), 4096)
        new = _log_int(rng, 1, max(1, new))
    window = rng.choice([0, 0, 0, _log_int(rng, 1, 8192)])
    return dict(kind=kind, B=B, Hq=H * G, H=H, d=d, P=P, cached=cached, new=new, ragged=rng.random() < 0.5,
                window=window, sinks=rng.choice([0, 1, 4, 100]) if window else 0, dtype=dtype,
                packed=rng.random() < 0.3)


# ---- inputs ------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _randn(shape, seed, salt, dtype):
    return torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _spread(n, b, B):
    """Request b's share of n in a ragged batch: odd numbers from about n / 8 up to n."""
    return max(1, n - (b * 7919 % B) * (7 * n // 8) // B - (b & 1))


def _new_cached(case):
    """New and cached tokens of every request (a ragged batch: every third one a single new token)."""
    B, new, cached = case["B"], case["new"], case["cached"]
    if not case["ragged"]:
        return [new] * B, [cached] * B
    return ([1 if b % 3 == 2 else _spread(new, b, B) for b in range(B)],
            [_spread(cached, (b * 5 + 1) % B, B) for b in range(B)])


def _tables(blocks, n_pages, most, seed, fill=0):
    """Tables int32 [B][most] of requests of so many pages, handed out in an arbitrary order, and the pages left."""
    order = torch.randperm(n_pages, generator=_gen(seed, 3), device="cuda").int()
    table = torch.full((len(blocks), most), fill, dtype=torch.int32, device="cuda")
    table[torch.arange(most, device="cuda") < _ints(blocks)[:, None]] = order[:sum(blocks)]
    return table, order[sum(blocks):]


def _pages(lens, P, seed):
    """The tables of requests of these lengths whose pages are all there are, and how many."""
    blocks = [(n + P - 1) // P for n in lens]
    return _tables(blocks, sum(blocks), max(blocks), seed)[0], sum(blocks)


def _pool(n_pages, H, P, d, dtype, seed):
    """Pages of keys (with a few large channels) and values, [n_pages][H][P][d]."""
    k = _randn((n_pages, H, P, d), seed, 11, DTYPES[dtype])
    k[..., 5::d // 4] *= 5
    return k, _randn((n_pages, H, P, d), seed, 13, DTYPES[dtype])


def _packed(n, heads, H, d, dtype, seed):
    """A packed projection of n tokens, [n][heads + 2 H][d]."""
    x = _randn((n, heads + 2 * H, d), seed, 17, DTYPES[dtype])
    return x[:, :heads], x[:, heads:heads + H], x[:, heads + H:]


def _plan_lengths(case):
    """Cached, kept (0: a new request in the place of another) and new tokens of every request."""
    B, new, every = case["B"], case["new"], case["replaced"]
    cached = [_spread(case["cached"], b, B) for b in range(B)]
    keep = [0 if every and b % every == 0 else n for b, n in enumerate(cached)]
    return cached, keep, [new if new == 1 else _spread(new, (b * 3 + 1) % B, B) for b in range(B)]


def prepare(case, seed):
    s = dict(case=case)
    kind, P = case["kind"], case["P"]
    if kind == "plan":
        B = case["B"]
        cached, keep, new = _plan_lengths(case)
        need = [(k + n + 2 * P) // P for k, n in zip(keep, new)]
        n_pages = sum((n + 2 * P) // P for n in cached) + sum(need)
        most = (case["cached"] + case["new"]) // P + 3
        g = torch.Generator()
        g.manual_seed(int(seed))
        shift = torch.randint(0, P, (B,), generator=g).tolist()     # other seeds end elsewhere in their pages
        cached = [n + m for n, m in zip(cached, shift)]
        keep = [0 if k == 0 else n for k, n in zip(keep, cached)]
        used = [(n + P - 1) // P for n in cached]
        table, left = _tables(used, n_pages, most, seed, fill=-1)
        free = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        free[:len(left)] = left
        n_slots = sum(new) if max(new) == 1 else (sum(new) + 1023) // 1024 * 1024
        s.update(table=table, free=free, state=_ints(cached + [len(left), 0]), keep=_ints(keep), new=_ints(new),
                 n_slots=n_slots, n_pages=n_pages, state_out=torch.zeros(B + 2, dtype=torch.int32, device="cuda"),
                 cu=torch.zeros(B + 1, dtype=torch.int32, device="cuda"), status=_ints([0]),
                 slots=torch.zeros(n_slots, dtype=torch.int32, device="cuda"))
        if own:     # the pages' contents are not looked at
            s["k"] = s["v"] = torch.empty((n_pages, 1, P, 64), dtype=torch.float16, device="cuda")
    elif kind == "write":
        n, H, d = case["n"], case["H"], case["d"]
        n_pages = (n + P - 1) // P + 3
        s["k"], s["v"] = _pool(n_pages, H, P, d, case["dtype"], seed)
        if case["packed"]:
            _, s["k_new"], s["v_new"] = _packed(n, 4 * H, H, d, case["dtype"], seed)
        else:
            s["k_new"], s["v_new"] = (_randn((n, H, d), seed, salt, DTYPES[case["dtype"]]) for salt in (5, 7))
        if n <= 1024:   # a decode step: single tokens anywhere
            slots = torch.randperm(n_pages * P, generator=_gen(seed, 3), device="cuda")[:n]
        else:           # a prompt: runs of a page
            pages = torch.randperm(n_pages, generator=_gen(seed, 3), device="cuda")
            slots = (pages[:, None] * P + torch.arange(P, device="cuda")).reshape(-1)[:n]
        s.update(slots=slots.int(), n_pages=n_pages, B=1, most=1)
    elif kind == "gather":
        B, H, d, n, first = (case[k] for k in ("B", "H", "d", "n", "first"))
        lens = [first + _spread(n, b, B) if B > 1 else first + n for b in range(B)]
        s["table"], n_pages = _pages(lens, P, seed)
        s["k"], s["v"] = _pool(n_pages, H, P, d, case["dtype"], seed)
        s["first"] = _ints([first] * B) if first else None
        s.update(state=_ints(lens + [0, 0]), n_pages=n_pages,
                 x_k=torch.zeros((B, H, n, d), dtype=torch.float16, device="cuda"),
                 x_v=torch.zeros((B, H, n, d), dtype=torch.float16, device="cuda"))
    else:
        B, Hq, H, d = (case[k] for k in ("B", "Hq", "H", "d"))
        new, cached = _new_cached(case)
        lens = [a + b for a, b in zip(new, cached)]
        s["table"], n_pages = _pages(lens, P, seed)
        s["k"], s["v"] = _pool(n_pages, H, P, d, case["dtype"], seed)
        if case["packed"]:
            s["q"] = _packed(sum(new), Hq, H, d, case["dtype"], seed)[0]
        else:
            s["q"] = _randn((sum(new), Hq, d), seed, 19, DTYPES[case["dtype"]])
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        s.update(cu=_ints(cu), state=_ints(lens + [0, 0]), n_pages=n_pages, max_q=max(new), max_tokens=max(lens),
                 out=torch.zeros((sum(new), Hq, d), dtype=DTYPES[case["dtype"]], device="cuda"))
    if own:
        import paper_2505_22913_amd as mf
        B = case.get("B", 1)
        s["cache"] = mf.PagedCache(B, s["k"].shape[1], s["k"].shape[3], s["n_pages"], P, k=s["k"], v=s["v"],
                                   table=s.get("table"), state=s.get("state"), free=s.get("free"),
                                   max_pages=s["table"].shape[1] if "table" in s else 1)
        if kind == "attend":
            need = mf.mustafar_paged_attn_workspace_bytes(s["cache"], case["Hq"], s["q"].shape[0], s["max_q"],
                                                          s["max_tokens"])
            s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------------------
def _plan(s):
    P, B, (table, free, n_slots) = s["case"]["P"], s["case"]["B"], (s["table"], s["free"], s["n_slots"])
    n_pages, most = s["n_pages"], table.shape[1]
    len0, n_free, new = s["state"][:B].long(), s["state"][B].long(), s["new"].long()
    kept = torch.minimum(s["keep"].long().clamp(min=0), len0)
    len1 = kept + new
    ob, nb = (len0 + P - 1) // P, (len1 + P - 1) // P
    grow, shrink = (nb - ob).clamp(min=0), (ob - nb).clamp(min=0)
    grown, shrunk = torch.cumsum(grow, 0), torch.cumsum(shrink, 0)
    A, R = grown[-1], shrunk[-1]
    cu = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    status = ((A - R > n_free).int() + 2 * (nb.max() > most).int() + 4 * (cu[-1] > n_slots).int()
              + 8 * ((new.min() < 0) | (len0.min() < 0) | (n_free < 0) | (n_free > n_pages)).int())
    j = torch.arange(most, device=table.device)
    # given up: into one list, row by row; a place behind it takes what is not
    gone = (j >= nb[:, None]) & (j < ob[:, None])
    at = torch.where(gone, (shrunk - shrink)[:, None] + j - nb[:, None], B * most)
    given = torch.zeros(B * most + 1, dtype=torch.int32, device=table.device)
    given = given.scatter(0, at.reshape(-1), torch.where(gone, table, 0).reshape(-1))
    # taken: first what was given up, then the top of the stack
    taken = (j >= ob[:, None]) & (j < nb[:, None])
    i = (grown - grow)[:, None] + j - ob[:, None]
    page = torch.where(i < R, given[i.clamp(0, B * most)], free[(n_free - 1 - (i - R)).clamp(0, n_pages - 1)])
    table = torch.where(taken, page, table)
    r = n_free + R - 1 - torch.arange(n_pages, device=table.device)   # which page given up lies at each place
    stack = torch.arange(n_pages, device=table.device)
    free = torch.where((stack >= n_free) & (stack < n_free + R - A), given[r.clamp(0, B * most)], free)
    t = torch.arange(n_slots, device=table.device)
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=B - 1)
    pos = (kept[b] + t - cu[b]).clamp(min=0)
    slots = table[b, (pos // P).clamp(max=most - 1)] * P + pos % P
    slots = torch.where(t < cu[-1], slots, -1)
    return dict(table=table, free=free, state=torch.cat([len1, (n_free + R - A)[None]]).int(), cu=cu.int(),
                slots=slots.int(), status=status[None].int())


def _write(s):
    P, slots = s["case"]["P"], s["slots"].long()
    s["k"][slots // P, :, slots % P] = s["k_new"]
    s["v"][slots // P, :, slots % P] = s["v_new"]
    return [s["k"], s["v"]]


def _tokens(s, first, n):
    """Page and place in it of tokens first[b] .. first[b] + n - 1 (long [B][n]), and whether they are there."""
    P, B, table = s["case"]["P"], s["case"]["B"], s["table"]
    tok = first + torch.arange(n, device=table.device).expand(B, n)
    there = tok < s["state"][:B].long()[:, None]
    return table.gather(1, torch.where(there, tok // P, 0)).long(), tok % P, there


def _gather(s):
    first = s["first"].long()[:, None] if s["first"] is not None else 0
    page, place, there = _tokens(s, first, s["case"]["n"])

    def dense(pool, x):
        y = pool[page, :, place].float().clamp(-65504, 65504).half().transpose(1, 2)
        return torch.where(there[:, None, :, None], y, x)

    return [dense(s["k"], s["x_k"]), dense(s["v"], s["x_v"])]


def _attend(s):
    case, cu = s["case"], s["cu"].long()
    B, Hq, H, d = (case[k] for k in ("B", "Hq", "H", "d"))
    G, nq, N = Hq // H, s["max_q"], s["max_tokens"]
    page, place, there = _tokens(s, 0, N)
    k, v = (s[x][page, :, place].transpose(1, 2).float() for x in ("k", "v"))      # [B][H][N][d]
    v = torch.where(there[:, None, :, None], v, 0.0)
    i = torch.arange(nq, device=cu.device)
    new = cu[1:] - cu[:-1]
    row = torch.where(i < new[:, None], cu[:-1, None] + i, 0)                      # [B][nq]
    q = s["q"][row].float().view(B, nq, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * nq, d)
    score = torch.matmul(q, k.transpose(2, 3)).div_(math.sqrt(d)).view(B, H, G, nq, N)
    pos = (s["state"][:B].long() - new)[:, None, None] + i[:, None]
    j = torch.arange(N, device=cu.device)
    sees = (j <= pos) & there[:, None]
    if case["window"]:
        sees &= (j > pos - case["window"]) | (j < case["sinks"])
    score.masked_fill_(~sees[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    o = torch.matmul(p.view(B, H, G * nq, N), v).view(B, H, G, nq, d) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, nq, Hq, d)
    t = torch.arange(s["q"].shape[0], device=cu.device)
    b = torch.searchsorted(cu[1:], t, right=True)
    return o[b, t - cu[b]].to(s["q"].dtype)


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"plan": _plan, "write": _write, "gather": _gather, "attend": _attend}[case["kind"]](s)
    import paper_2505_22913_amd as mf
    cache = s["cache"]
    if case["kind"] == "plan":
        mf.mustafar_paged_plan(cache, s["new"], s["n_slots"], keep=s["keep"], state_out=s["state_out"], cu=s["cu"],
                               slots=s["slots"], status=s["status"])
        return dict(table=cache.table, free=cache.free, state=s["state_out"][:case["B"] + 1], cu=s["cu"],
                    slots=s["slots"], status=s["status"])
    if case["kind"] == "write":
        mf.mustafar_paged_write(cache, s["k_new"], s["v_new"], s["slots"])
        return [cache.k, cache.v]
    if case["kind"] == "gather":
        return list(mf.mustafar_paged_gather(cache, case["n"], first=s["first"], x_k=s["x_k"], x_v=s["x_v"]))
    return mf.mustafar_paged_attn(s["q"], cache, s["cu"], max_q=s["max_q"], max_tokens=s["max_tokens"],
                                  window=case["window"], sinks=case["sinks"], out=s["out"], ws=s["ws"])


# ---- what a pass cannot do without -------------------------------------------------------------
def _seen(new, cached, window, sinks):
    """Cache tokens that some new token of a request sees, and pairs of a new token and one that it sees."""
    if not window:
        return new + cached, new * cached + new * (new + 1) // 2
    lo = max(0, cached - window + 1)
    tokens = new + cached - lo + min(sinks, lo)
    pos = torch.arange(cached, cached + new, dtype=torch.int64)
    near = torch.clamp(pos + 1, max=window)
    return tokens, int((near + torch.minimum(pos + 1 - near, torch.tensor(sinks))).sum())


def work(case):
    """Each input read once and each output written once; flops: the products of visible pairs."""
    kind = case["kind"]
    if kind == "plan":
        cached, keep, new = _plan_lengths(case)
        P = case["P"]
        pages = sum(abs((k + n + P - 1) // P - (c + P - 1) // P) for c, k, n in zip(cached, keep, new))
        return {"bytes": 4 * (5 * case["B"] + 2 * pages + sum(new) + sum(n // P + 1 for n in new)), "flops": 0}
    if kind == "write":
        return {"bytes": 8 * case["n"] * case["H"] * case["d"] + 4 * case["n"], "flops": 0}
    if kind == "gather":
        B, n = case["B"], case["n"]
        tokens = sum(_spread(n, b, B) for b in range(B)) if B > 1 else n
        return {"bytes": 8 * tokens * case["H"] * case["d"], "flops": 0}
    new, cached = _new_cached(case)
    seen = [_seen(a, b, case["window"], case["sinks"]) for a, b in zip(new, cached)]
    d = case["d"]
    return {"bytes": 4 * d * (case["H"] * sum(t for t, _ in seen) + case["Hq"] * sum(new)),
            "flops": 4 * d * case["Hq"] * sum(p for _, p in seen)}


# ---- the same outputs in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    """Whole numbers have no such value; the others are computed request by request."""
    kind, P = case["kind"], case["P"]
    if kind == "plan":
        return None
    H, d = case["H"], case["d"]
    if kind == "write":
        s = prepare(case, seed)
        for pool, x in (("k", "k_new"), ("v", "v_new")):
            flat = s[pool].double().transpose(1, 2).reshape(-1, H, d)      # [slot][H][d]
            flat[s["slots"].long()] = s[x].double()
            s[pool] = flat.view(-1, P, H, d).transpose(1, 2)
        return [s["k"], s["v"]]
    if kind == "gather":
        s = prepare(case, seed)
        out = [torch.zeros(s["x_k"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, L in enumerate(s["state"].tolist()[:case["B"]]):
            for x, pool in zip(out, (s["k"], s["v"])):
                rows = pool[s["table"][b, :(L + P - 1) // P].long()].double().transpose(0, 1).reshape(H, -1, d)
                x[b, :, :L - case["first"]] = rows[:, case["first"]:L]
        return out
    B, Hq, window, sinks = (case[k] for k in ("B", "Hq", "window", "sinks"))
    new, cached = _new_cached(case)
    if 4 * d * Hq * sum(a * (a + b) for a, b in zip(new, cached)) > PAIR_LIMIT:
        return None
    lens = [a + b for a, b in zip(new, cached)]
    table, n_pages = _pages(lens, P, seed)
    pool_k, pool_v = _pool(n_pages, H, P, d, case["dtype"], seed)
    if case["packed"]:
        q = _packed(sum(new), Hq, H, d, case["dtype"], seed)[0]
    else:
        q = _randn((sum(new), Hq, d), seed, 19, DTYPES[case["dtype"]])
    out = torch.empty((sum(new), Hq, d), dtype=torch.float64, device="cuda")
    at = 0
    for b, (a, L) in enumerate(zip(new, lens)):
        pages = table[b, :(L + P - 1) // P].long()
        far = torch.arange(L, device="cuda")[None] - torch.arange(L - a, L, device="cuda")[:, None]     # [a][L]
        hidden = far > 0
        if window:
            hidden |= (far <= -window) & (torch.arange(L, device="cuda") >= sinks)
        for h in range(H):
            k = pool_k[pages, h].reshape(-1, d)[:L].double()
            v = pool_v[pages, h].reshape(-1, d)[:L].double()
            for g in range(h * (Hq // H), (h + 1) * (Hq // H)):
                x = q[at:at + a, g].double() @ k.t() / d ** 0.5
                out[at:at + a, g] = torch.softmax(x.masked_fill(hidden, -torch.inf), -1) @ v
        at += a
    return out
