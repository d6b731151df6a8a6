"""What a decode step needs around the packed Linears and the 4-bit KV cache, as measurable cases: positions, scores, answers.

A program that serves a model rotates the rows of Q and K that the projection gave by their positions before K goes into the cache, attends
to the cache with the scores that its model was trained with (capped, biased by distance, with a prefix that all rows see), and reports
of the logits how likely the chosen tokens were.

  rope       ams_rope of the rows of Q and K of a call, halves or neighbours paired, part of a head or all of it, several scalings of the
             frequencies; `transposed`: the gradient's direction
  attention  ams_kv_attention over the 4-bit cache with softcap, slopes (a bias -slope |position - key|) or prefix_lens (keys that every
             row of the sequence sees)
  logprobs   ams_logprobs: log probability and rank of given tokens, entropy, the most likely tokens

Cache: uint8 [pages, kv_heads, block].  A block holds `page` tokens of a head in tiles of 16: first every tile's K codes, then the
V codes, the K scales, the V scales.  K codes of a tile: [plane][channels 8g..8g+7 of 32][token][word][byte], a word holding the
codes of 8 channels, low nibble first.  V codes: [plane][tokens 4q..4q+3][channel mod 16][word][token], a byte holding channels
16 (2w) + c and 16 (2w + 1) + c, the lower one in the low nibble for even tokens and in the high one for odd tokens.
K scales [token][run], V scales [tokens 4q..4q+3][run][token].
"""

from __future__ import annotations

import math

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of e2m1
WORKSPACE = 64 << 20  # bytes: as much as any call takes
HEADS = ((32, 8), (64, 8), (28, 4), (16, 16), (40, 40), (12, 1))  # query heads, kv heads
VOCABULARIES = (128256, 151936, 32000, 65536)
MAX_VALUES = 1 << 28  # kv_heads * tokens * dim of a drawn attention
MAX_PAIRS = 1 << 28  # heads * rows * keys of a drawn prompt
MAX_ROTATED = 16384 * 72 * 128  # values of a drawn rotation
MAX_LOGITS = 2048 * 128256  # of a drawn case


def listed():
    attention = dict(op="attention", softcap=0.0, bias=False, prefix=0, window=0, causal=True, lse=False)
    return [
        # one token of one sequence of an 8B model: the latency of a call
        dict(name="rope_first_token", op="rope", heads=32, kv_heads=8, dim=128, rot=128, base=500000.0, scaling="none", factor=1.0, trained=0, interleaved=False, transposed=False, batch=1, rows=1, tokens=18, ragged=False),
        # several prompts, wide heads of which a quarter is rotated, neighbours paired, a context four times the trained one
        dict(name="rope_ragged_part", op="rope", heads=16, kv_heads=16, dim=256, rot=64, base=10000.0, scaling="yarn", factor=4.0, trained=8192, interleaved=True, transposed=False, batch=9, rows=700, tokens=32011, ragged=True),
        # a prompt of a 70B model, far behind what is cached already, long wavelengths stretched
        dict(name="rope_prompt_70b", op="rope", heads=64, kv_heads=8, dim=128, rot=128, base=500000.0, scaling="bands", factor=8.0, trained=8192, interleaved=False, transposed=False, batch=1, rows=16384, tokens=120011, ragged=False),
        # one sequence that has just begun, capped scores, wide heads: the latency of a call
        dict(attention, name="cap_first_tokens", heads=16, kv_heads=8, dim=256, group=32, page=16, batch=1, rows=1, tokens=17, ragged=False, softcap=50.0),
        # a full batch of an 8B model with capped scores, every sequence at a length of its own, one slot idle
        dict(attention, name="cap_decode_8b", heads=32, kv_heads=8, dim=128, group=32, page=64, batch=32, rows=1, tokens=8192, ragged=True, softcap=30.0),
        # many short sequences with a bias by distance, a kv head to each query head
        dict(attention, name="bias_decode_short", heads=40, kv_heads=40, dim=128, group=128, page=32, batch=24, rows=1, tokens=1000, ragged=True, bias=True),
        # a chunk of a long prompt after what is there already, capped and biased
        dict(attention, name="cap_bias_prompt_8b", heads=32, kv_heads=8, dim=128, group=32, page=64, batch=1, rows=2048, tokens=8192, ragged=False, softcap=50.0, bias=True),
        # prompts of several lengths that begin with what all rows see (a picture, instructions), a sliding window behind it
        dict(attention, name="prefix_prompts_window", heads=16, kv_heads=16, dim=64, group=32, page=16, batch=7, rows=1999, tokens=1999, ragged=True, prefix=333, window=512, lse=True),
        # one sequence: the latency of a call
        dict(name="logprobs_token", op="logprobs", rows=1, vocab=128256, wide=False, top=5, temperature=1.0, allowed=1.0),
        # a full batch of an 8B model with what an interface reports
        dict(name="logprobs_step", op="logprobs", rows=32, vocab=128256, wide=False, top=20, temperature=0.7, allowed=1.0),
        # logits that a program has worked on, in 32 bits, most tokens ruled out by a grammar, an odd vocabulary
        dict(name="logprobs_masked", op="logprobs", rows=300, vocab=49999, wide=True, top=8, temperature=1.0, allowed=0.05),
        # the tokens of a prompt, scored
        dict(name="logprobs_prompt", op="logprobs", rows=2048, vocab=128256, wide=False, top=1, temperature=1.0, allowed=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rope", "attention", "attention", "logprobs"))
    if op == "logprobs":
        vocab = rng.choice(VOCABULARIES) if rng.random() < 0.4 else _log_int(rng, 100, 200000)
        wide = rng.random() < 0.4
        rows = _log_int(rng, 1, max(1, min(4096, MAX_LOGITS // (vocab * (2 if wide else 1)))))
        return dict(op=op, rows=rows, vocab=vocab, wide=wide, top=rng.choice((1, 1, 5, 20, rng.randint(2, 32))), temperature=rng.choice((1.0, 1.0, 0.6, 1.3)), allowed=rng.choice((1.0, 1.0, 0.9, 0.02)))
    heads, kv_heads = rng.choice(HEADS)
    dim = rng.choice((128, 128, 64, 256))
    while True:
        batch = _log_int(rng, 1, 64)
        tokens = _log_int(rng, 1, 131072)
        rows = min(tokens, rng.choice((1, 1, rng.randint(2, 16), _log_int(rng, 17, 8192))))
        if op == "rope":
            if batch * rows * (heads + kv_heads) * dim <= MAX_ROTATED:
                break
        elif batch * kv_heads * tokens * dim <= MAX_VALUES and batch * heads * rows * tokens <= MAX_PAIRS:
            break
    ragged = batch > 1 and rng.random() < 0.7
    if op == "rope":
        if rng.random() < 0.2:
            dim = rng.choice((80, 96, 112))  # heads that the cache has no kernels for
        scaling = rng.choice(("none", "none", "linear", "ntk", "yarn", "bands"))
        return dict(op=op, heads=heads, kv_heads=kv_heads, dim=dim, rot=rng.choice((dim, dim, dim // 2, dim // 4)), base=rng.choice((10000.0, 500000.0, 1000000.0)), scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0, 3.7)), trained=rng.choice((4096, 8192, 32768)), interleaved=rng.random() < 0.4, transposed=rng.random() < 0.2,
                    batch=batch, rows=rows, tokens=tokens, ragged=ragged)
    causal = rng.random() < 0.9
    kind = rng.choice(("cap", "bias", "prefix", "both", "all"))
    window = _log_int(rng, 8, 8192) if causal and rng.random() < 0.3 else 0
    return dict(op=op, heads=heads, kv_heads=kv_heads, dim=dim, group=rng.choice([g for g in (32, 32, 64, 128) if g <= dim]), page=rng.choice((16, 32, 64, 64, 128)), batch=batch, rows=rows, tokens=tokens,
                ragged=ragged, softcap=rng.choice((20.0, 30.0, 50.0)) if kind in ("cap", "both", "all") or not causal else 0.0, bias=kind in ("bias", "both", "all"),
                prefix=_log_int(rng, 1, tokens) if causal and kind in ("prefix", "all") else 0, window=window, causal=causal, lse=rng.random() < 0.3)


def _lengths(case):
    """(tokens, rows) of each sequence: lengths spread over the range, and an idle slot (no token, one row) in a large batch that decodes."""
    if not case["ragged"]:
        return [case["tokens"]] * case["batch"], [case["rows"]] * case["batch"]
    u = [(0.6180339887 * (b + 1)) % 1.0 for b in range(case["batch"])]
    tokens = [max(1, int(case["tokens"] * (0.1 + 0.9 * x))) for x in u]
    tokens[0] = case["tokens"]
    if case["rows"] == case["tokens"]:
        return tokens, tokens
    rows = [max(1, min(t, int(case["rows"] * (0.25 + 0.75 * ((x * 7.31) % 1.0))))) for t, x in zip(tokens, u)]
    if case["batch"] >= 8 and case["rows"] == 1:
        tokens[-1] = 0
    return tokens, rows


def _prefixes(case):
    """Keys that all rows of a sequence see: of different lengths, none for some."""
    return [min(t, int(case["prefix"] * ((0.37 * b) % 1.0 + 0.25))) if b % 4 != 2 else 0 for b, t in enumerate(_lengths(case)[0])]


def _generator(seed, i):
    return torch.Generator(device="cuda").manual_seed((seed * 1009 + i) % (1 << 62))


def _gains(case, seed):
    """Channels of K differ in size, as they do behind a trained projection."""
    return torch.exp(0.5 * torch.randn((case["kv_heads"], case["dim"]), generator=_generator(seed, 1), device="cuda"))


def _slopes(case):
    """A bias for each head, falling off by powers as it does in models that use it instead of rotary positions."""
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / case["heads"]) for h in range(case["heads"])], dtype=torch.float32)


def _page_count(case):
    return sum(-(-t // case["page"]) for t in _lengths(case)[0]) + 3


def _table(case, seed):
    """Pages of each sequence, in no order; entries that none belongs to are -1."""
    lens = _lengths(case)[0]
    order = torch.randperm(_page_count(case), generator=_generator(seed, 2), device="cuda").to(torch.int32)
    used = [-(-t // case["page"]) for t in lens]
    table = torch.full((case["batch"], max(used) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at : at + n]
        at += n
    return table


def _cached(case, seed):
    """Codes [2, pages * page, kv_heads, dim] of K and V and their scales [2, pages * page, kv_heads, runs], in the pool's order."""
    n, h, d, g = _page_count(case) * case["page"], case["kv_heads"], case["dim"], case["group"]
    codes = torch.empty((2, n, h, d), dtype=torch.uint8, device="cuda")
    scales = torch.empty((2, n, h, d // g), dtype=torch.float16, device="cuda")
    step = max(1, (1 << 26) // (h * d))
    for i in range(2):
        gen = _generator(seed, 3 + i)
        for at in range(0, n, step):
            x = torch.randn((min(step, n - at), h, d), generator=gen, device="cuda")
            if i == 0:
                x *= _gains(case, seed)
            codes[i, at : at + step], scales[i, at : at + step] = _quantized(x.half().float(), g)
    return codes, scales


def _quantized(x, group):
    """e2m1 codes of x [..., dim] (32 bits) and the fp16 scales [..., runs]."""
    run = x.unflatten(-1, (-1, group))
    scale = (run.abs().amax(-1) / 6).half()
    scale = torch.where(scale == 0, 1.0, scale)
    s = scale.float().unsqueeze(-1)
    size = run.abs()
    code = (size > 0.25 * s).to(torch.uint8)  # a tie goes to the even code
    for i, (level, up) in enumerate(zip(LEVELS[1:], LEVELS[2:])):
        middle = 0.5 * (level + up) * s
        code += (size >= middle) if i % 2 == 0 else (size > middle)
    code |= (run < 0).to(torch.uint8) << 3
    return code.flatten(-2), scale


def _words(case):
    return min(4, case["dim"] // 32)


def _laid_out(case, codes, scales):
    """The pool's bytes [pages, kv_heads, block]."""
    p, h, d, page, w = _page_count(case), case["kv_heads"], case["dim"], case["page"], _words(case)
    tiles, planes = page // 16, d // 32 // _words(case)
    k = codes[0].view(p, tiles, 16, h, planes, w, 4, 4, 2)  # page, tile, token, head, plane, word, g, byte, nibble
    k = k.permute(0, 3, 1, 4, 6, 2, 5, 7, 8)  # page, head, tile, plane, g, token, word, byte, nibble
    k = (k[..., 0] | (k[..., 1] << 4)).reshape(p, h, -1)
    v = codes[1].view(p, tiles, 4, 4, h, planes, w, 2, 16)  # page, tile, quad, token, head, plane, word, nibble, channel
    v = v.permute(0, 4, 1, 5, 2, 8, 6, 3, 7)  # page, head, tile, plane, quad, channel, word, token, nibble
    odd = (torch.arange(4, device="cuda") % 2 == 1).view(4)
    v = torch.where(odd, v[..., 1] | (v[..., 0] << 4), v[..., 0] | (v[..., 1] << 4)).reshape(p, h, -1)
    ks = scales[0].view(p, tiles, 16, h, -1).permute(0, 3, 1, 2, 4).reshape(p, h, -1).contiguous()
    vs = scales[1].view(p, tiles, 4, 4, h, -1).permute(0, 4, 1, 2, 5, 3).reshape(p, h, -1).contiguous()
    return torch.cat((k, v, ks.view(torch.uint8), vs.view(torch.uint8)), 2)


def _projected(case, seed):
    """Rows of Q and K as views of one projection's output [rows, heads + 2 kv_heads, dim]."""
    h, hk, d, total = case["heads"], case["kv_heads"], case["dim"], sum(_lengths(case)[1])
    x = torch.empty((total, h + 2 * hk, d), dtype=torch.float16, device="cuda")
    gen = _generator(seed, 5)
    for at in range(0, total, 4096):
        x[at : at + 4096] = torch.randn((min(4096, total - at), h + 2 * hk, d), generator=gen, device="cuda").half()
    return x[:, :h], x[:, h : h + hk]


def _logits(case, seed):
    """Logits of a trained model: bell-shaped, a few far above the rest, and where a grammar rules tokens out -inf."""
    rows, vocab = case["rows"], case["vocab"]
    x = torch.empty((rows, vocab), dtype=torch.float32 if case["wide"] else torch.float16, device="cuda")
    gen = _generator(seed, 6)
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    step = max(1, (1 << 26) // vocab)
    for at in range(0, rows, step):
        n = min(step, rows - at)
        y = 2.5 * torch.randn((n, vocab), generator=gen, device="cuda")
        likely = torch.randint(0, vocab, (n, 12), generator=gen, device="cuda")
        y.scatter_(1, likely, 9 + 2 * torch.randn((n, 12), generator=gen, device="cuda"))
        tokens[at : at + n] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.7, likely[:, 0], tokens[at : at + n])
        if case["allowed"] < 1:
            kept = torch.rand((n, vocab), generator=gen, device="cuda") < case["allowed"]
            kept.scatter_(1, tokens[at : at + n].unsqueeze(1), True)
            y = torch.where(kept, y, -math.inf)
        x[at : at + n] = y.to(x.dtype)
    return x, tokens.to(torch.int32)


def prepare(case, seed):
    if case["op"] == "logprobs":
        rows, top = case["rows"], case["top"]
        state = {"case": case}
        state["logits"], state["tokens"] = _logits(case, seed)
        if own:
            state["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
            reals, wholes = (lambda *n: torch.empty(n, dtype=torch.float32, device="cuda")), (lambda *n: torch.empty(n, dtype=torch.int32, device="cuda"))
            state["out"] = (reals(rows), wholes(rows), reals(rows), reals(rows, top), wholes(rows, top))
        return state
    h, d = case["heads"], case["dim"]
    tokens, rows = _lengths(case)
    total = sum(rows)
    state = {"case": case, "kv_lens": torch.tensor(tokens, dtype=torch.int32, device="cuda")}
    starts = torch.zeros(case["batch"] + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(rows).cumsum(0)
    state["q_starts"] = None if max(rows) == 1 else starts.cuda()
    state["rows"], state["max_rows"] = total, max(rows)
    state["q"], state["k"] = _projected(case, seed)
    if case["op"] == "rope":
        if own:
            import paper_2510_16045_amd as ams

            turns, state["magnitude"] = ams.ams_rope_frequencies(case["rot"], case["base"], case["scaling"], case["factor"], case["trained"])
            state["turns"] = torch.from_numpy(turns).cuda()
            state["out"] = tuple(torch.empty(x.shape, dtype=torch.float16, device="cuda") for x in (state["q"], state["k"]))
        return state
    state["table"] = _table(case, seed)
    state["cache"] = _laid_out(case, *_cached(case, seed))
    state["slopes"] = _slopes(case).cuda() if case["bias"] else None
    state["prefix_lens"] = torch.tensor(_prefixes(case), dtype=torch.int32, device="cuda") if case["prefix"] else None
    state["out"] = torch.empty((total, h, d), dtype=torch.float16, device="cuda")
    state["lse"] = torch.empty((total, h), dtype=torch.float32, device="cuda") if case["lse"] else None
    state["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    return state


def _row_places(state):
    """Sequence and position of every row of the call."""
    lens = state["kv_lens"].long()
    batch = lens.numel()
    starts = torch.arange(batch + 1, device="cuda") if state["q_starts"] is None else state["q_starts"].long()
    counts = starts[1:] - starts[:-1]
    seq = torch.repeat_interleave(torch.arange(batch, device="cuda"), counts, output_size=state["rows"])
    row = torch.arange(state["rows"], device="cuda") - starts[seq]
    return seq, row, lens[seq] - counts[seq] + row


def _frequencies(case):
    """Radians per position of each pair, and what rotated values are multiplied with."""
    r, base, factor, trained = case["rot"], case["base"], case["factor"], case["trained"]
    if case["scaling"] == "ntk":
        base *= factor ** (r / (r - 2))
    theta = [base ** (-2 * i / r) for i in range(r // 2)]
    if case["scaling"] == "linear":
        theta = [t / factor for t in theta]
    elif case["scaling"] == "bands":  # 1 to 4 turns within the trained length: from stretched to kept
        kept = [min(1.0, max(0.0, (trained * t / (2 * math.pi) - 1) / 3)) for t in theta]
        theta = [k * t + (1 - k) * t / factor for k, t in zip(kept, theta)]
    elif case["scaling"] == "yarn":  # pairs between those that make 32 turns and one within the trained length
        pair = [r * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (32, 1)]
        lo, hi = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), r - 1)
        kept = [1 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001))) for i in range(r // 2)]
        theta = [k * t + (1 - k) * t / factor for k, t in zip(kept, theta)]
        return theta, 0.1 * math.log(factor) + 1
    return theta, 1.0


def _plain_rope(state):
    case = state["case"]
    r = case["rot"]
    theta, magnitude = _frequencies(case)
    angle = _row_places(state)[2].double().unsqueeze(1) * torch.tensor(theta, dtype=torch.float64, device="cuda")
    c, s = (magnitude * torch.cos(angle)).float().unsqueeze(1), (magnitude * torch.sin(angle)).float().unsqueeze(1)
    if case["transposed"]:
        s = -s
    out = []
    for x in (state["q"], state["k"]):
        y = x.float()
        a, b = (y[..., :r:2], y[..., 1:r:2]) if case["interleaved"] else (y[..., : r // 2], y[..., r // 2 : r])
        pair = (a * c - b * s, b * c + a * s)
        turned = torch.stack(pair, -1).flatten(-2) if case["interleaved"] else torch.cat(pair, -1)
        out.append(torch.cat((turned, y[..., r:]), -1).half())
    return out


def _values(codes, scales):
    """fp16 values, as 32 bits, of nibbles [..., dim] with their scales [..., runs]."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device="cuda")
    x = level[codes.int()].unflatten(-1, (scales.shape[-1], -1))
    return (x * scales.float().unsqueeze(-1)).half().float().flatten(-2)


def _restored(case, blocks):
    """K and V [..., page, dim] of blocks [..., bytes]."""
    d, page, w, runs = case["dim"], case["page"], _words(case), case["dim"] // case["group"]
    tiles, planes = page // 16, d // 32 // w
    lead = blocks.shape[:-1]
    n = len(lead)
    kc, vc, ks, vs = blocks.split((page * d // 2, page * d // 2, page * runs * 2, page * runs * 2), -1)
    order = lambda t, axes: t.permute(*range(n), *(n + a for a in axes))  # noqa: E731
    k = torch.stack((kc & 15, kc >> 4), -1).view(*lead, tiles, planes, 4, 16, w, 4, 2)
    k = order(k, (0, 3, 1, 4, 2, 5, 6)).reshape(*lead, page, d)
    v = torch.stack((vc & 15, vc >> 4), -1).view(*lead, tiles, planes, 4, 16, w, 4, 2)
    odd = (torch.arange(4, device="cuda") % 2 == 1).view(4, 1)
    v = torch.where(odd, v.flip(-1), v)
    v = order(v, (0, 2, 5, 1, 4, 6, 3)).reshape(*lead, page, d)
    ks = ks.contiguous().view(torch.float16).view(*lead, page, runs)
    vs = order(vs.contiguous().view(torch.float16).view(*lead, tiles, 4, runs, 4), (0, 1, 3, 2)).reshape(*lead, page, runs)
    return _values(k, ks), _values(v, vs)


def _plain_attention(state):
    case = state["case"]
    h, hk, d, batch, most = case["heads"], case["kv_heads"], case["dim"], case["batch"], state["max_rows"]
    seq, row, position = _row_places(state)
    k, v = _restored(case, state["cache"][state["table"].clamp(min=0).long()])
    k = k.transpose(1, 2).flatten(2, 3)  # [batch, kv_heads, keys, dim]
    v = v.transpose(1, 2).flatten(2, 3)
    q = torch.zeros((batch, most, h, d), device="cuda")
    q[seq, row] = state["q"].float()
    at = torch.full((batch, most), -1, dtype=torch.long, device="cuda")
    at[seq, row] = position
    q = q.view(batch, most, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(batch, hk, -1, d)
    s = (q @ k.transpose(-1, -2).contiguous()).view(batch, hk, h // hk, most, -1)
    s = s * (1 / math.sqrt(d))
    if case["softcap"]:
        s = case["softcap"] * torch.tanh(s / case["softcap"])
    key = torch.arange(k.shape[2], device="cuda")
    if case["bias"]:
        far = (at.unsqueeze(-1) - key).abs().float().view(batch, 1, 1, most, -1)
        s = s - state["slopes"].view(1, hk, h // hk, 1, 1) * far
    there = (key < state["kv_lens"].view(-1, 1)).unsqueeze(1)  # [batch, rows, keys]
    allowed = there
    if case["causal"]:
        allowed = allowed & (key <= at.unsqueeze(-1))
    if case["window"]:
        allowed = allowed & (key > at.unsqueeze(-1) - case["window"])
    if case["prefix"]:
        allowed = allowed | (there & (key < state["prefix_lens"].view(-1, 1, 1)))
    allowed = allowed.view(batch, 1, 1, allowed.shape[1], -1)
    s = torch.where(allowed, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total == 0, 1.0, total)).view(batch, hk, -1, p.shape[-1])
    o = (p @ v).view(batch, hk, h // hk, most, d).permute(0, 3, 1, 2, 4).reshape(batch, most, h, d)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(batch, most, h)
    return (o[seq, row].half(), lse[seq, row]) if case["lse"] else o[seq, row].half()


def _plain_logprobs(state):
    case = state["case"]
    raw = state["logits"].float()
    rows, vocab = raw.shape
    place = torch.arange(vocab, device="cuda")
    token = state["tokens"].long().unsqueeze(1)
    given = raw.gather(1, token)
    rank = ((raw > given) | ((raw == given) & (place < token))).sum(1)
    x = raw * (1 / case["temperature"])
    x = x - x.amax(1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    entropy = torch.log(total) - torch.where(e > 0, e * x, 0.0).sum(1, keepdim=True) / total
    x = x - torch.log(total)
    tokens = torch.empty((rows, case["top"]), dtype=torch.long, device="cuda")
    left = raw.clone()
    taken = torch.zeros_like(raw, dtype=torch.bool)
    for i in range(case["top"]):  # of equal logits the first
        best = left.amax(1, keepdim=True)
        tokens[:, i] = torch.where((left == best) & ~taken, place, vocab).amin(1).clamp(max=vocab - 1)
        left.scatter_(1, tokens[:, i : i + 1], -math.inf)
        taken.scatter_(1, tokens[:, i : i + 1], True)
    return x.gather(1, token).squeeze(1), rank.to(torch.int32), entropy.squeeze(1), x.gather(1, tokens), tokens.to(torch.int32)


def run(state):
    case = state["case"]
    if not own:
        return {"rope": _plain_rope, "attention": _plain_attention, "logprobs": _plain_logprobs}[case["op"]](state)
    import paper_2510_16045_amd as ams

    if case["op"] == "rope":
        return list(ams.ams_rope(state["q"], state["k"], state["turns"], kv_lens=state["kv_lens"], q_starts=state["q_starts"], magnitude=state["magnitude"], interleaved=case["interleaved"],
                                 transposed=case["transposed"], out=state["out"]))
    if case["op"] == "attention":
        ams.ams_kv_attention(state["q"], state["cache"], state["table"], state["kv_lens"], case["group"], q_starts=state["q_starts"], max_q_len=state["max_rows"], causal=case["causal"], window=case["window"],
                             workspace=state["workspace"], out=state["out"], lse=state["lse"], softcap=case["softcap"], slopes=state["slopes"], prefix_lens=state["prefix_lens"])
        return (state["out"], state["lse"]) if case["lse"] else state["out"]
    return tuple(ams.ams_logprobs(state["logits"], state["tokens"], top=case["top"], temperature=case["temperature"], workspace=state["workspace"], out=state["out"]))


def _pairs(case):
    """(row, key) pairs of one head, and the keys of a sequence that some row attends to, summed over the sequences."""
    pairs = keys = 0
    for t, n, prefix in zip(*_lengths(case), _prefixes(case) if case["prefix"] else [0] * case["batch"]):
        if t == 0:
            continue
        if not case["causal"]:
            pairs, keys = pairs + n * t, keys + t
            continue
        win = case["window"] or t
        for p in range(t - n, t):
            begin = max(p + 1 - win, 0)
            pairs += p + 1 - begin + max(prefix - p - 1, 0) + min(prefix, begin)
        begin = max(t - n + 1 - win, 0)
        keys += t - begin + min(prefix, begin)
    return pairs, keys


def work(case):
    if case["op"] == "logprobs":
        values = case["rows"] * case["vocab"]
        return {"bytes": values * (4 if case["wide"] else 2) + case["rows"] * (16 + 8 * case["top"]), "flops": 4 * values}
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    rows = sum(_lengths(case)[1])
    if case["op"] == "rope":
        return {"bytes": 4 * rows * (h + hk) * d, "flops": 3 * rows * (h + hk) * case["rot"]}
    held = hk * (d + 4 * (d // case["group"]))  # bytes of a token's K and V in the cache
    pairs, keys = _pairs(case)
    return {"bytes": keys * held + 4 * rows * h * d + (4 * rows * h if case["lse"] else 0), "flops": 4.0 * d * h * pairs}


def exact(case, seed):
    if case["op"] == "logprobs":
        logits, tokens = _logits(case, seed)
        rows, vocab = logits.shape
        out = [[] for _ in range(5)]
        step = max(1, (1 << 26) // vocab)
        for at in range(0, rows, step):
            raw, token = logits[at : at + step], tokens[at : at + step].long()
            order = torch.sort(raw.float(), dim=1, descending=True, stable=True)[1]
            lp = torch.log_softmax(raw.double() / case["temperature"], 1)
            best = order[:, : case["top"]]
            out[0].append(lp.gather(1, token.view(-1, 1)).view(-1))
            out[1].append((order == token.view(-1, 1)).int().argmax(1).to(torch.int32))
            out[2].append(-torch.where(lp == -math.inf, 0.0, lp * lp.exp()).sum(1))
            out[3].append(lp.gather(1, best))
            out[4].append(best.to(torch.int32))
        return tuple(torch.cat(x) for x in out)
    tokens, rows = _lengths(case)
    if case["op"] == "rope":
        r = case["rot"]
        theta, magnitude = _frequencies(case)
        w = torch.tensor(theta, dtype=torch.float64, device="cuda") * (-1 if case["transposed"] else 1)
        position = torch.cat([torch.arange(t - n, t, device="cuda") for t, n in zip(tokens, rows)]).double()
        first = torch.arange(r // 2, device="cuda") * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else r // 2)
        out = []
        for x in _projected(case, seed):
            y = x.double()
            for at in range(0, y.shape[0], 1024):
                turn = magnitude * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), position[at : at + 1024, None] * w)
                z = torch.complex(y[at : at + 1024, :, first], y[at : at + 1024, :, second]) * turn.unsqueeze(1)
                y[at : at + 1024, :, first], y[at : at + 1024, :, second] = z.real, z.imag
            out.append(y)
        return out
    h, hk, d, g = case["heads"], case["kv_heads"], case["dim"], case["group"]
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    codes, scales = _cached(case, seed)
    table = _table(case, seed).long()
    place = torch.arange(case["page"], device="cuda")
    slopes = _slopes(case).double().tolist()
    prefixes = _prefixes(case) if case["prefix"] else [0] * case["batch"]

    def held(b, i, head, t):  # values of sequence b's first t tokens of one head
        at = (table[b, : -(-t // case["page"])].unsqueeze(1) * case["page"] + place).flatten()[:t]
        c, s = codes[i][at][:, head].long(), scales[i][at][:, head].double()
        x = level[c & 7] * (1 - 2 * (c >> 3)) * s.repeat_interleave(g, -1)
        return x.half().double()

    q = _projected(case, seed)[0]
    out = torch.zeros((sum(rows), h, d), dtype=torch.float64, device="cuda")
    lse = torch.full((sum(rows), h), -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for b, (t, n) in enumerate(zip(tokens, rows)):
        if t:
            i, j = torch.arange(t - n, t, device="cuda").unsqueeze(1), torch.arange(t, device="cuda")
            barred = torch.zeros((n, t), dtype=torch.bool, device="cuda")
            if case["causal"]:
                barred |= j > i
            if case["window"]:
                barred |= j <= i - case["window"]
            barred &= j >= prefixes[b]
            for head in range(h):
                if head % (h // hk) == 0:
                    k, v = (held(b, which, head // (h // hk), t) for which in range(2))
                s = (q[at : at + n, head].double() @ k.t()) / math.sqrt(d)
                if case["softcap"]:
                    s = torch.tanh(s / case["softcap"]) * case["softcap"]
                if case["bias"]:
                    s -= slopes[head] * (i - j).abs()
                s.masked_fill_(barred, -math.inf)
                out[at : at + n, head] = torch.softmax(s, -1) @ v
                lse[at : at + n, head] = torch.logsumexp(s, -1)
        at += n
    return (out, lse) if case["lse"] else out
