"""The operators of the 4-bit KV cache as measurable cases: writing rows into it, reading them back, attention over it.

A program that serves a model quantized with AMS-Quant keeps the keys and values of its sequences in pages of FP4-e2m1 codes
with one fp16 scale per run of channels.  Each step it writes the rows of K and V that the Linears gave (one per sequence, or a
prompt's), and attends to the cache with the rows of Q; a prefix that is moved or reused is read back.

  write      ams_kv_write of new rows, and ams_kv_read of the same rows (their values as the cache holds them)
  read       ams_kv_read of whole sequences
  attention  ams_kv_attention of the last rows of each sequence (one: decoding; a few: drafts; many: prompts)

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
MAX_VALUES = 1 << 28  # kv_heads * tokens * dim of a drawn case
MAX_PAIRS = 1 << 28  # heads * rows * keys of a drawn prompt


def listed():
    return [
        # one sequence of an 8B model that has just begun: the latency of a call
        dict(name="decode_first_tokens", op="attention", heads=32, kv_heads=8, dim=128, group=32, page=16, batch=1, rows=1, tokens=17, ragged=False, causal=True, window=0, lse=False),
        # a full batch of an 8B model, every sequence at a length of its own, one slot idle
        dict(name="decode_8b_batch", op="attention", heads=32, kv_heads=8, dim=128, group=32, page=64, batch=32, rows=1, tokens=8192, ragged=True, causal=True, window=0, lse=False),
        # one sequence at the longest context
        dict(name="decode_8b_long", op="attention", heads=32, kv_heads=8, dim=128, group=64, page=64, batch=1, rows=1, tokens=131071, ragged=False, causal=True, window=0, lse=True),
        # many short sequences, seven query heads to a kv head, one scale per row
        dict(name="decode_short_batch", op="attention", heads=28, kv_heads=4, dim=128, group=128, page=32, batch=64, rows=1, tokens=1000, ragged=True, causal=True, window=0, lse=False),
        # drafts of five tokens checked at once on a 70B model
        dict(name="draft_70b", op="attention", heads=64, kv_heads=8, dim=128, group=32, page=128, batch=16, rows=5, tokens=3001, ragged=False, causal=True, window=0, lse=False),
        # a chunk of a long prompt after what is there already
        dict(name="prompt_chunk_8b", op="attention", heads=32, kv_heads=8, dim=128, group=32, page=64, batch=1, rows=2048, tokens=8192, ragged=False, causal=True, window=0, lse=False),
        # prompts of several lengths, with a sliding window and narrow heads
        dict(name="prompts_window", op="attention", heads=16, kv_heads=16, dim=64, group=32, page=16, batch=7, rows=1999, tokens=1999, ragged=True, causal=True, window=512, lse=True),
        # the rows of one decode step of a full batch
        dict(name="write_step", op="write", heads=32, kv_heads=8, dim=128, group=32, page=64, batch=32, rows=1, tokens=8192, ragged=True, causal=True, window=0, lse=False),
        # a prompt of a 70B model
        dict(name="write_prompt", op="write", heads=64, kv_heads=8, dim=128, group=32, page=64, batch=1, rows=16384, tokens=20011, ragged=False, causal=True, window=0, lse=False),
        # several prompts, wide heads
        dict(name="write_ragged", op="write", heads=16, kv_heads=16, dim=256, group=64, page=32, batch=9, rows=700, tokens=900, ragged=True, causal=True, window=0, lse=False),
        # a shared prefix of a few sequences
        dict(name="read_prefix", op="read", heads=32, kv_heads=8, dim=128, group=128, page=16, batch=5, rows=333, tokens=333, ragged=True, causal=True, window=0, lse=False),
        # the whole cache of a long sequence, to be moved
        dict(name="read_long", op="read", heads=32, kv_heads=8, dim=128, group=32, page=64, batch=1, rows=131072, tokens=131072, ragged=False, causal=True, window=0, lse=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "write", "read"))
    heads, kv_heads = rng.choice(HEADS)
    dim = rng.choice((128, 128, 64, 256))
    group = rng.choice([g for g in (32, 32, 64, 128) if g <= dim])
    kind = rng.choice(("one", "one", "few", "many")) if op != "read" else "all"
    while True:
        batch = _log_int(rng, 1, 64)
        tokens = _log_int(rng, 1, 131072)
        rows = {"one": 1, "few": rng.randint(2, 16), "many": _log_int(rng, 17, 8192), "all": tokens}[kind]
        rows = min(rows, tokens)
        if batch * kv_heads * tokens * dim <= MAX_VALUES and (op != "attention" or batch * heads * rows * tokens <= MAX_PAIRS):
            break
    causal = op != "attention" or rng.random() < 0.85
    window = _log_int(rng, 8, 8192) if op == "attention" and causal and rng.random() < 0.25 else 0
    return dict(op=op, heads=heads, kv_heads=kv_heads, dim=dim, group=group, page=rng.choice((16, 32, 64, 64, 128)), batch=batch, rows=rows, tokens=tokens,
                ragged=batch > 1 and rng.random() < 0.7, causal=causal, window=window, lse=op == "attention" and rng.random() < 0.3)


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


def _generator(seed, i):
    return torch.Generator(device="cuda").manual_seed((seed * 1009 + i) % (1 << 62))


def _gains(case, seed):
    """Channels of K differ in size, as they do behind a trained projection."""
    return torch.exp(0.5 * torch.randn((case["kv_heads"], case["dim"]), generator=_generator(seed, 1), device="cuda"))


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
    most = run.abs().amax(-1)
    scale = (most / 6).half()
    scale = torch.where(scale == 0, 1.0, scale)
    scale = torch.where(torch.isfinite(most), scale, math.nan)
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


def prepare(case, seed):
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    tokens, rows = _lengths(case)
    total = sum(rows)
    state = {"case": case, "table": _table(case, seed), "kv_lens": torch.tensor(tokens, dtype=torch.int32, device="cuda")}
    state["cache"] = _laid_out(case, *_cached(case, seed))
    starts = torch.zeros(case["batch"] + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(rows).cumsum(0)
    state["q_starts"] = None if max(rows) == 1 else starts.cuda()
    state["rows"], state["max_rows"] = total, max(rows)
    if case["op"] == "read":
        state["out"] = tuple(torch.empty((total, hk, d), dtype=torch.float16, device="cuda") for _ in range(2))
        return state
    q, k, v = _projected(case, seed)
    state["q"], state["k"], state["v"] = q, k, v
    if case["op"] == "write":
        state["out"] = tuple(torch.empty((total, hk, d), dtype=torch.float16, device="cuda") for _ in range(2))
    else:
        state["out"] = torch.empty((total, h, d), dtype=torch.float16, device="cuda")
        state["lse"] = torch.empty((total, h), dtype=torch.float32, device="cuda") if case["lse"] else None
        state["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    return state


def _projected(case, seed):
    """Rows of Q, K and V as views of one projection's output."""
    h, hk, d, total = case["heads"], case["kv_heads"], case["dim"], sum(_lengths(case)[1])
    x = torch.randn((total, h + 2 * hk, d), generator=_generator(seed, 5), device="cuda")
    x[:, h : h + hk] *= _gains(case, seed)
    x = x.half()
    return x[:, :h], x[:, h : h + hk], x[:, h + hk :]


def _row_places(state):
    """Sequence and position of every row of the call."""
    lens = state["kv_lens"].long()
    batch = lens.numel()
    starts = torch.arange(batch + 1, device="cuda") if state["q_starts"] is None else state["q_starts"].long()
    counts = starts[1:] - starts[:-1]
    seq = torch.repeat_interleave(torch.arange(batch, device="cuda"), counts, output_size=state["rows"])
    row = torch.arange(state["rows"], device="cuda") - starts[seq]
    return seq, row, lens[seq] - counts[seq] + row


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


def _places(state, seq, position):
    """Where the rows at `position` of `seq` lie: bytes of K's and of V's codes [rows, kv_heads, dim / 2] and halves of their scales [rows, kv_heads, runs]."""
    case = state["case"]
    hk, d, page, w, runs = case["kv_heads"], case["dim"], case["page"], _words(case), case["dim"] // case["group"]
    number = state["table"][seq, position // page].long()
    block = (number.view(-1, 1) * hk + torch.arange(hk, device="cuda")).unsqueeze(2) * state["cache"].shape[-1]
    at = position % page
    tile, token = (at // 16).view(-1, 1), (at % 16).view(-1, 1)
    pair = torch.arange(d // 2, device="cuda")
    i, g, byte = pair // 16, pair // 4 % 4, pair % 4  # K: channels 2j, 2j + 1
    k = tile * 8 * d + i // w * 256 * w + (g * 16 + token) * 4 * w + i % w * 4 + byte
    c = pair % 16  # V: channels 32 i + c, 32 i + 16 + c
    v = page * d // 2 + tile * 8 * d + i // w * 256 * w + (token // 4 * 16 + c) * 4 * w + i % w * 4 + token % 4
    run = torch.arange(runs, device="cuda")
    ks = page * d + 2 * ((tile * 16 + token) * runs + run)
    vs = page * (d + 2 * runs) + 2 * (((tile * 4 + token // 4) * runs + run) * 4 + token % 4)
    return [block + k.unsqueeze(1), block + v.unsqueeze(1), (block + ks.unsqueeze(1)) // 2, (block + vs.unsqueeze(1)) // 2]


def _plain_read(state):
    seq, _, position = _row_places(state)
    odd, there = (position % 2 == 1).view(-1, 1, 1, 1), (position >= 0).view(-1, 1, 1)
    flat = state["cache"].view(-1)
    kc, vc, ks, vs = _places(state, seq, position.clamp(min=0))
    k, v, half = flat[kc], flat[vc], flat.view(torch.float16)
    k = torch.stack((k & 15, k >> 4), -1).flatten(-2)
    v = torch.stack((v & 15, v >> 4), -1)
    v = torch.where(odd, v.flip(-1), v).unflatten(-2, (-1, 16)).transpose(-1, -2).flatten(-3)
    return [torch.where(there, x, 0.0).half() for x in (_values(k, half[ks]), _values(v, half[vs]))]


def _plain_write(state):
    case = state["case"]
    seq, _, position = _row_places(state)
    fits = position >= 0
    kw, vw, ksw, vsw = _places(state, seq[fits], position[fits])
    kc, ks = _quantized(state["k"][fits].float(), case["group"])
    vc, vs = _quantized(state["v"][fits].float(), case["group"])
    flat = state["cache"].view(-1)
    flat[kw] = kc[..., ::2] | (kc[..., 1::2] << 4)
    pair = vc.unflatten(-1, (-1, 2, 16))
    low, high = pair[..., 0, :].flatten(-2), pair[..., 1, :].flatten(-2)
    odd = (position[fits] % 2 == 1).view(-1, 1, 1)
    flat[vw] = torch.where(odd, high | (low << 4), low | (high << 4))
    half = flat.view(torch.float16)
    half[ksw], half[vsw] = ks, vs


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
    key = torch.arange(k.shape[2], device="cuda")
    allowed = (key < state["kv_lens"].view(-1, 1)).unsqueeze(1)  # [batch, rows, keys]
    if case["causal"]:
        allowed = allowed & (key <= at.unsqueeze(-1))
    if case["window"]:
        allowed = allowed & (key > at.unsqueeze(-1) - case["window"])
    allowed = allowed.view(batch, 1, 1, allowed.shape[1], -1)
    s = torch.where(allowed, s * (1 / math.sqrt(d)), -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total == 0, 1.0, total)).view(batch, hk, -1, p.shape[-1])
    o = (p @ v).view(batch, hk, h // hk, most, d).permute(0, 3, 1, 2, 4).reshape(batch, most, h, d)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(batch, most, h)
    return (o[seq, row].half(), lse[seq, row]) if case["lse"] else o[seq, row].half()


def run(state):
    case = state["case"]
    if not own:
        if case["op"] == "attention":
            return _plain_attention(state)
        if case["op"] == "write":
            _plain_write(state)
        return _plain_read(state)
    import paper_2510_16045_amd as ams

    group, cache, table, lens, starts = case["group"], state["cache"], state["table"], state["kv_lens"], state["q_starts"]
    if case["op"] == "attention":
        ams.ams_kv_attention(state["q"], cache, table, lens, group, q_starts=starts, max_q_len=state["max_rows"], causal=case["causal"], window=case["window"],
                             workspace=state["workspace"], out=state["out"], lse=state["lse"])
        return (state["out"], state["lse"]) if case["lse"] else state["out"]
    if case["op"] == "write":
        ams.ams_kv_write(cache, state["k"], state["v"], table, lens, group, q_starts=starts)
    return list(ams.ams_kv_read(cache, table, lens, group, case["dim"], q_starts=starts, out=state["out"]))


def _pairs(case):
    """(row, key) pairs of one head, and the keys of a sequence that some row attends to, summed over the sequences."""
    pairs = keys = 0
    for t, n in zip(*_lengths(case)):
        if t == 0:
            continue
        if not case["causal"]:
            pairs, keys = pairs + n * t, keys + t
            continue
        win = case["window"] or t
        # the row at position p has min(p + 1, win) keys
        first = t - n
        short = max(0, min(t, win) - first)  # rows that see fewer keys than the window, or just it
        pairs += sum(range(first + 1, first + short + 1)) + (n - short) * min(win, t)
        keys += min(t, n - 1 + win)
    return pairs, keys


def work(case):
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    held = hk * (d + 4 * (d // case["group"]))  # bytes of a token's K and V in the cache
    rows = sum(_lengths(case)[1])
    if case["op"] == "attention":
        pairs, keys = _pairs(case)
        return {"bytes": keys * held + 4 * rows * h * d + (4 * rows * h if case["lse"] else 0), "flops": 4.0 * d * h * pairs}
    moved = rows * (held + 4 * hk * d)  # read back
    if case["op"] == "write":
        moved *= 2
    return {"bytes": moved, "flops": 0}


def exact(case, seed):
    tokens, rows = _lengths(case)
    h, hk, d, g = case["heads"], case["kv_heads"], case["dim"], case["group"]
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")

    def rounded(x):  # what the cache holds for x [..., dim]
        y = torch.empty_like(x, dtype=torch.float64)
        for c in range(0, d, g):
            part = x[..., c : c + g].double()
            most = part.abs().amax(-1, keepdim=True)
            s = (most / 6).half().double()
            s[s == 0] = 1.0
            off = (part.abs().unsqueeze(-1) - s.unsqueeze(-1) * level).abs()
            off[..., 1::2] += off[..., 1::2] * 1e-12  # of two that are as near the even code is taken
            y[..., c : c + g] = (level[off.argmin(-1)] * part.sign() * s).half().double()
        return y

    if case["op"] == "write":
        _, k, v = _projected(case, seed)
        step = max(1, (1 << 23) // (hk * d))
        there = torch.tensor([t - n + i >= 0 for t, n in zip(tokens, rows) for i in range(n)], dtype=torch.float64, device="cuda").view(-1, 1, 1)
        return [torch.cat([rounded(x[i : i + step]) for i in range(0, x.shape[0], step)]) * there for x in (k, v)]
    codes, scales = _cached(case, seed)
    table = _table(case, seed).long()
    place = torch.arange(case["page"], device="cuda")

    def held(b, i, head, t):  # values of sequence b's first t tokens of one head, or of all of them
        at = (table[b, : -(-t // case["page"])].unsqueeze(1) * case["page"] + place).flatten()[:t]
        c, s = codes[i][at][:, head].long(), scales[i][at][:, head].double()
        x = level[c & 7] * (1 - 2 * (c >> 3)) * s.repeat_interleave(g, -1)
        return x.half().double()

    if case["op"] == "read":
        return [torch.cat([held(b, i, slice(None), t)[t - n :] for b, (t, n) in enumerate(zip(tokens, rows))]) for i in range(2)]
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
            for head in range(h):
                if head % (h // hk) == 0:
                    k, v = (held(b, which, head // (h // hk), t) for which in range(2))
                s = (q[at : at + n, head].double() @ k.t()) / math.sqrt(d)
                s.masked_fill_(barred, -math.inf)
                out[at : at + n, head] = torch.softmax(s, -1) @ v
                lse[at : at + n, head] = torch.logsumexp(s, -1)
        at += n
    return (out, lse) if case["lse"] else out
