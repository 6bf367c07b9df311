"""Rotary positions and the paged cache of 8-bit codes, as cases that can be timed and compared.

A case is a dict of plain values; `kind` names the operator:

  rope    rotary positions of a step's queries and keys (`mustafar_rope`): halves or interleaved
          pairs, all of a head's channels or its first ones, rates for long contexts, and the
          rotation back, which is the gradient
  write   keys and values of new tokens into their pages as 8-bit codes with a power of two for
          each block of tokens and head (`mustafar_paged8_write`), and the blocks that the step
          touched read back (`mustafar_paged8_gather`)
  gather  requests' pages as the dense fp16 tensors that the compression takes
          (`mustafar_paged8_gather`)
  attend  causal attention of every request's new tokens over its pages of codes, with or without
          a sliding window and first tokens that stay visible (`mustafar_paged8_attn`)

`own` selects the library's kernels; without it every operator is computed with elementary torch
operations in 32 bits (angles in 64). Sizes are those of the library's synthetic workloads
(layers of 8 or 32 kv-heads, 1 to 8 query heads each, one sequence of 4K tokens to batches of 16K
and 32K) and of the steps of a serving loop.
"""
import math

import torch

own = False     # the library's kernels instead of the plain forms

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
PAIR_LIMIT = 1 << 42    # products of 64-bit pairs above which the exact answer takes too long


def listed():
    return [
        # A decode step of 64 running requests, positions from the cache's lengths: latency.
        dict(name="rope_decode_b64", kind="rope", B=64, new=1, Hq=32, H=8, d=128, rot=128, layout="half", scaling="plain",
             base=10000.0, at=8192, by="cache", packed=True, inverse=False, dtype="fp16"),
        # A large prompt step of a model with interleaved pairs and rates for eight times its
        # context, read out of the packed projection.
        dict(name="rope_prompt_16k_interleaved_bf16", kind="rope", B=16, new=1024, Hq=32, H=8, d=128, rot=128,
             layout="interleaved", scaling="turns", base=500000.0, at=100000, by="positions", packed=True, inverse=False,
             dtype="bf16"),
        # A training step's gradient through a rotation of a part of odd size of every head.
        dict(name="rope_back_4k_part_of_80", kind="rope", B=1, new=4096, Hq=32, H=32, d=80, rot=20, layout="half",
             scaling="plain", base=10000.0, at=0, by="positions", packed=False, inverse=True, dtype="bf16"),
        # The keys and values of a decode step: most fall into a block that holds older tokens.
        dict(name="write_decode_b64_e4m3", kind="write", B=64, cached=2048, new=1, ragged=True, H=8, d=128, P=64, block=16,
             code="e4m3", dtype="fp16", packed=False),
        # A large prompt step of several requests, out of the packed projection.
        dict(name="write_prompt_16k_int8_bf16", kind="write", B=8, cached=200, new=4096, ragged=True, H=8, d=128, P=16,
             block=16, code="int8", dtype="bf16", packed=True),
        # One short prompt on its way to the compressed cache.
        dict(name="gather_b1_mha_1k_int8", kind="gather", B=1, H=32, d=128, P=64, block=32, n=1000, first=0, code="int8",
             dtype="fp16"),
        # A batch of long prompts of a bf16 model, read back as the compressed caches' fp16.
        dict(name="gather_b8_gqa_16k_e4m3_bf16", kind="gather", B=8, H=8, d=128, P=64, block=16, n=16384, first=0,
             code="e4m3", dtype="bf16"),
        # One chat sequence of 4K tokens on a 32-head layer: the latency of a single call.
        dict(name="attend_decode_b1_mha_4k_e4m3", kind="attend", B=1, Hq=32, H=32, d=128, P=64, block=16, cached=4095, new=1,
             ragged=False, window=0, sinks=0, code="e4m3", dtype="fp16", packed=False),
        # A continuous batch of different lengths on a grouped-query layer with small pages.
        dict(name="attend_decode_b16_gqa4_16k_ragged_int8", kind="attend", B=16, Hq=32, H=8, d=128, P=16, block=16,
             cached=16384, new=1, ragged=True, window=0, sinks=0, code="int8", dtype="bf16", packed=False),
        # Long sequences of which each token sees the newest 1024 and four first ones.
        dict(name="attend_decode_b32_gqa8_d64_32k_window", kind="attend", B=32, Hq=64, H=8, d=64, P=32, block=32,
             cached=32768, new=1, ragged=False, window=1024, sinks=4, code="e4m3", dtype="bf16", packed=False),
        # A chunk of a long prompt whose first 16K tokens are in the cache.
        dict(name="attend_chunk_512_of_16k_gqa4_int8", kind="attend", B=1, Hq=32, H=8, d=128, P=64, block=64, cached=16384,
             new=512, ragged=False, window=0, sinks=0, code="int8", dtype="fp16", packed=False),
        # Whole prompts on a 32-head layer: the largest amount of arithmetic.
        dict(name="attend_prompts_b4_mha_4k_e4m3_bf16", kind="attend", B=4, Hq=32, H=32, d=128, P=64, block=16, cached=0,
             new=4096, ragged=False, window=0, sinks=0, code="e4m3", dtype="bf16", packed=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope"] * 3 + ["write"] * 2 + ["gather"] + ["attend"] * 5)
    dtype, code = rng.choice(["fp16", "bf16"]), rng.choice(["e4m3", "int8"])
    if kind == "rope":
        d = rng.choice([64, 80, 96, 128, 128, 256])
        H = rng.choice([1, 2, 4, 8, 8, 16, 32])
        G = rng.choice([1, 2, 3, 4, 8])
        B = _log_int(rng, 1, 256)
        most = 16384 * 40 * 128 // (B * H * (G + 1) * d)
        return dict(kind=kind, B=B, new=_log_int(rng, 1, max(1, min(16384, most))), Hq=H * G, H=H, d=d,
                    rot=rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["plain", "linear", "base", "turns"]), base=rng.choice([10000.0, 500000.0]),
                    at=_log_int(rng, 1, 1 << 20), by=rng.choice(["cache", "positions"]), packed=rng.random() < 0.5,
                    inverse=rng.random() < 0.3, dtype=dtype)
    P, d, H = rng.choice([16, 32, 64, 64, 128, 256]), rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 8, 8, 16, 32])
    block = rng.choice([n for n in (16, 32, 64) if n <= P])
    common = dict(kind=kind, H=H, d=d, P=P, block=block, code=code, dtype=dtype)
    if kind == "write":
        B = _log_int(rng, 1, 128)
        most = 16384 * 1024 // (B * H * d)
        cached = _log_int(rng, 1, max(1, min(4096, 32 * most)))
        new = rng.choice([1, _log_int(rng, 2, max(2, min(8192, most)))])
        return dict(common, B=B, cached=cached, new=new, ragged=rng.random() < 0.5, packed=rng.random() < 0.5)
    if kind == "gather":
        B = _log_int(rng, 1, 16)
        n = _log_int(rng, 1, max(1, min(32768, (1 << 27) // (B * H * d))))
        return dict(common, B=B, n=n, first=rng.choice([0, 0, rng.randint(1, 4096)]))
    G = rng.choice([1, 2, 3, 4, 4, 7, 8])
    B = _log_int(rng, 1, 32)
    most = (1 << 28) // (B * H * d)     # cached tokens per request
    cached = _log_int(rng, 1, max(1, min(65536, most)))
    new = 1
    if rng.random() < 0.6:
        # the scores of a whole batch, and fewer products than the largest listed case
        heads = B * H * G
        new = min((1 << 28) // (heads * cached), math.isqrt((1 << 36) // (heads * d)), (1 << 28) // (heads * d), 4096)
        new = _log_int(rng, 1, max(1, new))
    window = rng.choice([0, 0, 0, _log_int(rng, 1, 8192)])
    return dict(common, B=B, Hq=H * G, cached=cached, new=new, ragged=rng.random() < 0.5, window=window,
                sinks=rng.choice([0, 1, 4, 100]) if window else 0, packed=rng.random() < 0.3)


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


def _starts(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return cu


def _pages(lens, P, seed):
    """Tables of requests of these lengths, pages handed out in an arbitrary order, and the number of pages."""
    blocks = [(n + P - 1) // P for n in lens]
    order = torch.randperm(sum(blocks), generator=_gen(seed, 3), device="cuda").int()
    table = torch.zeros((len(lens), max(blocks)), dtype=torch.int32, device="cuda")
    table[torch.arange(max(blocks), device="cuda") < _ints(blocks)[:, None]] = order
    return table, sum(blocks)


def _tokens_of(shape, seed, salt, dtype, keys):
    """Keys (with a few large channels) or values of [..][d]."""
    x = _randn(shape, seed, salt, DTYPES[dtype])
    if keys:
        x[..., 5::shape[-1] // 4] *= 5
    return x


def _packed(n, Hq, H, d, dtype, seed):
    """A packed projection of n tokens, [n][Hq + 2 H][d]."""
    x = _randn((n, Hq + 2 * H, d), seed, 17, DTYPES[dtype])
    x[:, Hq:Hq + H, 5::d // 4] *= 5
    return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]


def _rates(case):
    """Radians per position of every pair, and the factor of the rotated channels."""
    rot, base, scaling = case["rot"], case["base"], case["scaling"]
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    if scaling == "base" and rot > 2:
        base *= 8.0 ** (rot / (rot - 2))
    rates = base ** (-i / rot)
    if scaling == "linear":
        rates = rates / 8
    if scaling == "turns":      # pairs that turn less than once in 8192 tokens are slowed down eight times
        keep = ((8192 * rates / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        rates = rates * (keep + (1 - keep) / 8)
    return rates.cuda(), 0.1 * math.log(8) + 1 if scaling == "turns" else 1.0


# ---- codes: a value is code * 2^(scale - 127), one scale byte for a block of tokens and head ---------
# (the largest magnitude that is held, the largest code's exponent and mantissa's complement, the least scale)
_HELD = {("e4m3", "fp16"): 61440.0, ("e4m3", "bf16"): 240 * 2.0 ** 120, ("int8", "fp16"): 65024.0, ("int8", "bf16"): 127 * 2.0 ** 121}
_TOP = {"e4m3": (8, 0x1fffff), "int8": (6, 0x01ffff)}
_LEAST = {("e4m3", "fp16"): 127 - 15, ("int8", "fp16"): 127 - 24, ("e4m3", "bf16"): 127 - 110, ("int8", "bf16"): 127 - 110}


def _held(case, x):
    most = _HELD[case["code"], case["dtype"]]
    return x.float().clamp(-most, most)


def _scale_of(case, top):
    """The least power of two, as its byte, that takes magnitudes up to `top` (fp32) to codes."""
    exponent, complement = _TOP[case["code"]]
    byte = (top.view(torch.int32) + complement >> 23) - exponent
    return byte.clamp(min=_LEAST[case["code"], case["dtype"]])


def _power(byte):
    return (byte.int() << 23).view(torch.float32)


def _encode(case, x):
    """fp32 in units of the scale to codes, to the nearest, ties to even."""
    if case["code"] == "e4m3":
        return x.to(torch.float8_e4m3fn)
    return x.round().to(torch.int8)


def _pool(case, n_pages, seed):
    """Pages of codes [n_pages][H][P][d] and scale bytes [n_pages][H][P / block], keys and values."""
    H, P, d, T = (case[k] for k in ("H", "P", "d", "block"))
    made = []
    for salt in (11, 13):
        codes = torch.empty((n_pages, H, P, d), dtype=CODES[case["code"]], device="cuda")
        scale = torch.empty((n_pages, H, P // T), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (H * P * d))
        for at in range(0, n_pages, step):
            n = min(step, n_pages - at)
            x = _held(case, _tokens_of((n, H, P, d), seed, salt + 100 * (at // step), case["dtype"], salt == 11))
            byte = _scale_of(case, x.view(n, H, P // T, T * d).abs().amax(-1))
            codes[at:at + n] = _encode(case, x / _power(byte).repeat_interleave(T, 2)[..., None])
            scale[at:at + n] = byte.to(torch.uint8)
        made += [codes, scale]
    return made


def prepare(case, seed):
    s = dict(case=case)
    kind, H, d, dtype = case["kind"], case["H"], case["d"], DTYPES[case["dtype"]]
    if kind == "rope":
        B, Hq = case["B"], case["Hq"]
        new = [case["new"] if B < 3 else _spread(case["new"], b, B) for b in range(B)]
        first = [_spread(case["at"], (b * 5 + 1) % B, B) if case["at"] else 0 for b in range(B)]
        n = sum(new)
        if case["packed"]:
            s["q"], s["k"], _ = _packed(n, Hq, H, d, case["dtype"], seed)
        else:
            s["q"], s["k"] = _randn((n, Hq, d), seed, 5, dtype), _tokens_of((n, H, d), seed, 7, case["dtype"], True)
        s["rates"], s["magnitude"] = _rates(case)
        s["out_q"] = torch.zeros((n, Hq, d), dtype=dtype, device="cuda")
        s["out_k"] = torch.zeros((n, H, d), dtype=dtype, device="cuda")
        s["cu"], s["state"] = _ints(_starts(new)), _ints([a + b for a, b in zip(new, first)] + [0, 0])
        s["positions"] = (torch.repeat_interleave(_ints(first) - s["cu"][:-1], _ints(new)) + torch.arange(n, device="cuda")).int()
    else:
        P, B = case["P"], case["B"]
        if kind == "gather":
            lens = [case["first"] + (_spread(case["n"], b, B) if B > 1 else case["n"]) for b in range(B)]
        else:
            new, cached = _new_cached(case)
            lens = [a + b for a, b in zip(new, cached)]
            s["cu"], s["max_q"], s["max_tokens"] = _ints(_starts(new)), max(new), max(lens)
        s["table"], n_pages = _pages(lens, P, seed)
        s["k"], s["k_scale"], s["v"], s["v_scale"] = _pool(case, n_pages, seed)
        s.update(state=_ints(lens + [0, 0]), n_pages=n_pages)
        if kind == "write":
            n = sum(new)
            if case["packed"]:
                _, s["k_new"], s["v_new"] = _packed(n, 4 * H, H, d, case["dtype"], seed)
            else:
                s["k_new"], s["v_new"] = (_tokens_of((n, H, d), seed, salt, case["dtype"], salt == 5) for salt in (5, 7))
            # from the start of the first block that the step touches
            s["first"], s["n"] = _ints([c // case["block"] * case["block"] for c in cached]), max(new) + case["block"]
        elif kind == "gather":
            s["first"], s["n"] = _ints([case["first"]] * B) if case["first"] else None, case["n"]
        else:
            Hq = case["Hq"]
            n = sum(new)
            s["q"] = _packed(n, Hq, H, d, case["dtype"], seed)[0] if case["packed"] else _randn((n, Hq, d), seed, 19, dtype)
            s["out"] = torch.zeros((n, Hq, d), dtype=dtype, device="cuda")
        if kind != "attend":
            s["x_k"], s["x_v"] = (torch.zeros((B, H, s["n"], d), dtype=torch.float16, device="cuda") for _ in range(2))
    if own:
        import paper_2505_22913_amd as mf
        if kind == "rope":
            scaling = case["scaling"] if case["scaling"] != "base" or case["rot"] > 2 else "plain"
            s["rope"] = mf.Rope(case["rot"], case["base"], case["layout"], scaling, factor=8.0, original_len=8192,
                                low_turns=1.0, high_turns=32.0, magnitude=s["magnitude"])
            if case["by"] == "cache":
                s["cache"] = mf.PagedCache(case["B"], 1, 64, 1, 1024, state=s["state"], max_pages=(1 << 21) // 1024)
        else:
            s["cache"] = mf.PagedCache8(case["B"], H, d, s["n_pages"], P, dtype=dtype, block_tokens=case["block"], k=s["k"],
                                        v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"], table=s["table"],
                                        state=s["state"])
        if kind == "attend":
            need = mf.mustafar_paged8_attn_workspace_bytes(s["cache"], case["Hq"], s["q"].shape[0], s["max_q"],
                                                           s["max_tokens"])
            s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------------------
def _rope(s):
    case, rot = s["case"], s["case"]["rot"]
    angle = s["positions"].double()[:, None] * s["rates"]
    c, t = (torch.cos(angle) * s["magnitude"]).float()[:, None], (torch.sin(angle) * s["magnitude"]).float()[:, None]
    if case["inverse"]:
        t = -t

    def turn(x):
        y = x.float()
        if case["layout"] == "half":
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            z = [a * c - b * t, a * t + b * c]
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            z = [torch.stack([a * c - b * t, a * t + b * c], -1).flatten(-2)]
        return torch.cat(z + [y[..., rot:]], -1).to(x.dtype)

    return [turn(s["q"]), turn(s["k"])]


def _slot(s, b, pos):
    """Slots of positions of requests."""
    P = s["case"]["P"]
    return s["table"][b, pos // P].long() * P + pos % P


def _write(s):
    case, cu, B = s["case"], s["cu"].long(), s["case"]["B"]
    P, T, H, d = (case[k] for k in ("P", "block", "H", "d"))
    t = torch.arange(s["k_new"].shape[0], device=cu.device)
    b = torch.searchsorted(cu[1:], t, right=True)
    first = s["state"][:B].long() - (cu[1:] - cu[:-1])          # position of every request's first new token
    slot = _slot(s, b, first[b] + t - cu[b])
    page, block, place = slot // P, slot % P // T, slot % P
    # the block that holds the token before the first new one, and its tokens up to there
    start = first // T * T
    rows = torch.arange(T, device=cu.device)
    old_slot = _slot(s, torch.arange(B, device=cu.device)[:, None], start[:, None] + rows)          # [B][T]
    old_page, old_place, old_block = old_slot // P, old_slot % P, old_slot[:, 0] % P // T
    older = (start[:, None] + rows < first[:, None])[..., None, None]
    for x_new, codes, scale in ((s["k_new"], s["k"], s["k_scale"]), (s["v_new"], s["v"], s["v_scale"])):
        x = _held(case, x_new)
        top = torch.zeros((s["n_pages"] * (P // T), H), device=cu.device)
        top.index_reduce_(0, page * (P // T) + block, x.abs().amax(-1), "amax")
        byte = _scale_of(case, top).view(-1, P // T, H).transpose(1, 2)                     # [n_pages][H][P / T]
        before = scale[old_page[:, 0], :, old_block].int()                                  # [B][H]
        byte[old_page[:, 0], :, old_block] = torch.maximum(byte[old_page[:, 0], :, old_block],
                                                           torch.where((start < first)[:, None], before, 0))
        scale[page, :, block] = byte[page, :, block].to(torch.uint8)
        old = codes.view(torch.uint8)[old_page, :, old_place].view(codes.dtype)             # [B][T][H][d]
        now = _encode(case, old.float() * _power((before - scale[old_page[:, 0], :, old_block].int() + 127).clamp(min=1))[:, None, :, None])
        codes.view(torch.uint8)[old_page, :, old_place] = torch.where(older, now.view(torch.uint8), old.view(torch.uint8))
        codes.view(torch.uint8)[page, :, place] = _encode(case, x / _power(byte[page, :, block])[..., None]).view(torch.uint8)
    return _gather(s) + [s["k_scale"], s["v_scale"]]


def _tokens(s, first, n):
    """Page and place in it of tokens first[b] .. first[b] + n - 1 (long [B][n]), and whether they are there."""
    P, B, table = s["case"]["P"], s["case"]["B"], s["table"]
    tok = first + torch.arange(n, device=table.device).expand(B, n)
    there = tok < s["state"][:B].long()[:, None]
    return table.gather(1, torch.where(there, tok // P, 0)).long(), tok % P, there


def _values(s, codes, scale, page, place):
    """Values of tokens, fp32 [B][H][n][d]."""
    x = codes.view(torch.uint8)[page, :, place].view(codes.dtype).float()
    return (x * _power(scale[page, :, place // s["case"]["block"]])[..., None]).transpose(1, 2)


def _gather(s):
    page, place, there = _tokens(s, 0 if s["first"] is None else s["first"].long()[:, None], s["n"])

    def dense(codes, scale, x):
        y = _values(s, codes, scale, page, place).clamp(-65504, 65504).half()
        return torch.where(there[:, None, :, None], y, x)

    return [dense(s["k"], s["k_scale"], s["x_k"]), dense(s["v"], s["v_scale"], s["x_v"])]


def _attend(s):
    case, cu = s["case"], s["cu"].long()
    B, Hq, H, d = (case[k] for k in ("B", "Hq", "H", "d"))
    G, nq, N = Hq // H, s["max_q"], s["max_tokens"]
    page, place, there = _tokens(s, 0, N)
    k, v = (_values(s, s[x], s[x + "_scale"], page, place) for x in ("k", "v"))    # [B][H][N][d]
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
        return {"rope": _rope, "write": _write, "gather": _gather, "attend": _attend}[case["kind"]](s)
    import paper_2505_22913_amd as mf
    if case["kind"] == "rope":
        where = dict(cache=s["cache"], cu=s["cu"]) if case["by"] == "cache" else dict(positions=s["positions"])
        return list(mf.mustafar_rope(s["rope"], s["q"], s["k"], **where, inverse=case["inverse"], out_q=s["out_q"],
                                     out_k=s["out_k"]))
    cache = s["cache"]
    if case["kind"] == "attend":
        return mf.mustafar_paged8_attn(s["q"], cache, s["cu"], max_q=s["max_q"], max_tokens=s["max_tokens"],
                                       window=case["window"], sinks=case["sinks"], out=s["out"], ws=s["ws"])
    if case["kind"] == "write":
        mf.mustafar_paged8_write(cache, s["k_new"], s["v_new"], s["cu"])
    x = list(mf.mustafar_paged8_gather(cache, s["n"], first=s["first"], x_k=s["x_k"], x_v=s["x_v"]))
    return x + [cache.k_scale, cache.v_scale] if case["kind"] == "write" else x


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
    """Each input read once and each output written once; flops: a rotation's, and the products of visible pairs."""
    kind, B, H, d = case["kind"], case["B"], case["H"], case["d"]
    if kind == "rope":
        n = sum(case["new"] if B < 3 else _spread(case["new"], b, B) for b in range(B))
        heads = n * (case["Hq"] + H)
        return {"bytes": 4 * heads * d + 4 * n, "flops": 3 * heads * case["rot"]}
    row = 2 * H * d     # of keys and values
    if kind == "gather":
        tokens = sum(_spread(case["n"], b, B) for b in range(B)) if B > 1 else case["n"]
        return {"bytes": 3 * row * tokens + 2 * H * tokens // case["block"], "flops": 0}
    new, cached = _new_cached(case)
    if kind == "write":
        back = sum(new) + sum(c % case["block"] for c in cached)    # tokens that are read back
        return {"bytes": row * (3 * sum(new) + 3 * back) + 6 * H * (back // case["block"] + B), "flops": 0}
    seen = [_seen(a, b, case["window"], case["sinks"]) for a, b in zip(new, cached)]
    tokens = sum(t for t, _ in seen)
    return {"bytes": row * tokens + 2 * H * tokens // case["block"] + 4 * d * case["Hq"] * sum(new),
            "flops": 4 * d * case["Hq"] * sum(p for _, p in seen)}


# ---- the same outputs in 64 bits ---------------------------------------------------------------
def _two_to(e):
    """2^e in float64, exactly, of whole numbers e."""
    return torch.tensor([2.0 ** k for k in range(-300, 301)], dtype=torch.float64, device=e.device)[e.long() + 300]


def _exact_values(case, codes, scale, table, L):
    """Values of a request's first L tokens, float64 [H][L][d]."""
    P, T = case["P"], case["block"]
    pages = table[:(L + P - 1) // P].long()
    power = _two_to(scale[pages].int() - 127).unsqueeze(-1).expand(-1, -1, -1, T).flatten(2)     # [pages][H][P]
    return (codes[pages].double() * power[..., None]).transpose(0, 1).flatten(1, 2)[:, :L]


def _exact_rope(case, seed):
    s = prepare(case, seed)
    rot = case["rot"]
    turn = torch.polar(torch.full((), float(s["magnitude"]), dtype=torch.float64, device="cuda"),
                       torch.outer(s["positions"].double(), s["rates"]))[:, None]
    turn = turn.conj() if case["inverse"] else turn
    out = []
    for x in (s["q"], s["k"]):
        y = x.double()
        pairs = y[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else y[..., :rot].unflatten(-1, (-1, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y[..., :rot] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
        out.append(y)
    return out


def _exact_held(case, x, before, older):
    """A block's values [n][H][d] after a write (float64) and its exponents [H], from its older tokens' values
    (the first `older`) with the exponents `before` and the new ones."""
    code, top = case["code"], {"e4m3": 448.0, "int8": 127.0}[case["code"]]
    most = _HELD[code, case["dtype"]]
    x = x.clamp(-most, most)
    part, e = torch.frexp(x[older:].abs().amax((0, 2)).clamp(min=1e-300) / top)
    e = (e - (part == 0.5).int()).clamp(min=_LEAST[code, case["dtype"]] - 127)
    if older:
        e = torch.maximum(e, before)
    unit = _two_to(e)[:, None]
    if code == "e4m3":      # 3 bits behind the leading one, none below 2^-9
        low = torch.frexp((x / unit).abs().clamp(min=2.0 ** -6)).exponent - 1
        unit = unit * _two_to(low - 3)
    return torch.round(x / unit) * unit, e


def _exact_write(case, seed):
    """The blocks that a step touches, one by one; as many as can be done in a few seconds."""
    H, d, P, T, B = (case[k] for k in ("H", "d", "P", "block", "B"))
    new, cached = _new_cached(case)
    if sum((n + T - 1) // T + 1 for n in new) > 4096:
        return None
    s = prepare(case, seed)
    out, at = [torch.zeros(s["x_k"].shape, dtype=torch.float64, device="cuda") for _ in range(2)], 0
    for b, (n, c) in enumerate(zip(new, cached)):
        L, lo = n + c, c // T * T
        for i, x in enumerate(("k", "v")):
            held = _exact_values(case, s[x], s[x + "_scale"], s["table"][b], L)[:, lo:c].transpose(0, 1)
            x_all = torch.cat([held, s[x + "_new"][at:at + n].double()])
            before = s[x + "_scale"][s["table"][b, lo // P].long(), :, lo % P // T].int() - 127
            for j in range(0, L - lo, T):
                older = max(0, min(T, c - lo - j))
                out[i][b, :, j:j + T][:, :L - lo - j] = _exact_held(case, x_all[j:j + T], before, older)[0].transpose(0, 1)
        at += n
    return out + [None, None]


def exact(case, seed):
    """Whole numbers have no such value; the others are computed request by request."""
    kind, B, H, d = case["kind"], case["B"], case["H"], case["d"]
    if kind == "rope":
        return _exact_rope(case, seed)
    if kind == "write":
        return _exact_write(case, seed)
    s = prepare(case, seed)
    lens = s["state"].tolist()[:B]
    if kind == "gather":
        out = [torch.zeros(s["x_k"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, L in enumerate(lens):
            for x, name in zip(out, ("k", "v")):
                x[b, :, :L - case["first"]] = _exact_values(case, s[name], s[name + "_scale"], s["table"][b], L)[:, case["first"]:]
        return out
    Hq, window, sinks = (case[k] for k in ("Hq", "window", "sinks"))
    new, cached = _new_cached(case)
    if 4 * d * Hq * sum(a * (a + b) for a, b in zip(new, cached)) > PAIR_LIMIT:
        return None
    out = torch.empty((sum(new), Hq, d), dtype=torch.float64, device="cuda")
    at = 0
    for b, (a, L) in enumerate(zip(new, lens)):
        k, v = (_exact_values(case, s[x], s[x + "_scale"], s["table"][b], L) for x in ("k", "v"))
        far = torch.arange(L, device="cuda")[None] - torch.arange(L - a, L, device="cuda")[:, None]     # [a][L]
        hidden = far > 0
        if window:
            hidden |= (far <= -window) & (torch.arange(L, device="cuda") >= sinks)
        for g in range(Hq):
            h = g // (Hq // H)
            x = s["q"][at:at + a, g].double() @ k[h].t() / d ** 0.5
            out[at:at + a, g] = torch.softmax(x.masked_fill(hidden, -torch.inf), -1) @ v[h]
        at += a
    return out
