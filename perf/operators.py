"""Chunks of new tokens over the packed cache, as calls that can be timed and checked: where their
tokens go (pages and slots, from the request lengths), the append of their keys and values, their
attention over the paged cache, and single-token attention through a sliding window with sinks.

A case is one such call.  `run` makes it through the library where `own` is true and computes the same
in elementary torch operations where it is not.  The packed cache is made here with plain torch, from
keys with outlier channels under RoPE.  Packed codes are compared as they lie in memory: the format
defines every bit of them (angle edges and fp16 parameters included).
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
PAIRS = HEAD_DIM // 2
GROUP = 128                    # tokens of a page
DEVICE = "cuda:0"

# ---- cases -----------------------------------------------------------------------------------


def _case(name, op, seqs, kv_heads, context, new, **more):
    case = dict(name=name, op=op, seqs=seqs, q_heads=4 * kv_heads, kv_heads=kv_heads, context=context, min_context=context,
                new=new, min_new=new, r_bits=4, t_bits=4, grouped_angles=False, v_bits=16, dtype="f16", tail=True, window=0,
                sinks=0, free=1.0)
    case.update(more)
    return case


def listed():
    return [
        # before every step of continuous batching: one more token each, most of them in the page they have
        _case("plan_step", "plan", 64, 8, 16384, 1, min_context=1024),
        # prompts of all sizes come in at once, some behind a conversation that is cached already
        _case("plan_prompts", "plan", 200, 8, 8192, 4096, min_context=0, min_new=1),
        # one step of a ragged batch: one key and one value row each
        _case("append_step", "append", 31, 8, 3000, 1, min_context=200),
        # chunks of a few prompts that begin and end inside pages, values quantized
        _case("append_chunks_v4", "append", 9, 8, 8000, 2048, min_context=0, min_new=300, v_bits=4),
        # whole prompts of fp32 keys at low bits
        _case("append_prompts_f32", "append", 2, 8, 0, 16384, min_new=16000, r_bits=3, t_bits=3, dtype="f32"),
        # drafted tokens of a batch are verified: five queries a sequence
        _case("chunk_verify", "chunk", 16, 8, 6000, 5, min_context=500),
        # a chunk of a long document: the largest call
        _case("chunk_long", "chunk", 1, 8, 32768, 2048),
        # chunks of one token to several hundred in one call, low bits, values quantized
        _case("chunk_ragged_v4", "chunk", 12, 8, 8192, 700, min_context=0, min_new=1, r_bits=3, t_bits=3, v_bits=4),
        # chunks of a model with a sliding window and sinks
        _case("chunk_window", "chunk", 2, 8, 16000, 2048, min_context=9000, window=1024, sinks=4),
        # one user of such a model, far into a conversation: latency counts
        _case("window_one", "window", 1, 8, 20000, 0, window=1024, sinks=4),
        # a serving batch of it
        _case("window_batch", "window", 32, 8, 32768, 0, min_context=4096, window=4096, sinks=4),
        # odd windows, sinks that end inside a second page, sequences shorter than the window, values quantized
        _case("window_ragged_v4", "window", 48, 8, 12000, 0, min_context=20, window=2001, sinks=130, v_bits=4),
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["plan"] * 2 + ["append"] * 3 + ["chunk"] * 4 + ["window"] * 4)
    r_bits, t_bits = rng.choice([(4, 4), (4, 4), (3, 3), (3, 3), (5, 3), (3, 5), (4, 2), (2, 4)])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 32])
    group = rng.choice([1, 2]) if kv_heads == 32 else rng.choice([1, 2, 3, 4, 4, 4, 6, 7, 8, 12, 16])
    case = _case(None, op, 1, kv_heads, 0, 0, q_heads=kv_heads * group, r_bits=r_bits, t_bits=t_bits,
                 grouped_angles=rng.random() < 0.25, v_bits=rng.choice([16, 16, 16, 4, 2]), tail=rng.random() < 0.75)
    del case["name"]
    if op == "plan":
        case.update(seqs=_log_uniform(rng, 1, 2000), context=_log_uniform(rng, 1, 32768), free=rng.choice([1.0, 1.0, 0.7]))
        case["new"] = _log_uniform(rng, 1, max(1, min(16384, 800000 // case["seqs"])))
    elif op == "append":
        case.update(dtype=rng.choice(["f16", "f16", "f32"]), tail=True)
        case["seqs"] = _log_uniform(rng, 1, 64)
        case["new"] = _log_uniform(rng, 1, max(1, min(16384, 260000 // (kv_heads * case["seqs"]))))
        case["context"] = _log_uniform(rng, 1, 8192)
    elif op == "chunk":
        # query heads x new tokens x context of the padded batch, up to the largest listed case's
        most = math.exp(rng.uniform(math.log(32 * 5 * 500), math.log(32 * 2048 * 34816)))
        case["seqs"] = _log_uniform(rng, 1, 32)
        rows = max(1.0, most / (case["q_heads"] * case["seqs"]))
        case["new"] = _log_uniform(rng, 1, max(1, min(4096, int(math.sqrt(rows)))))
        tokens = min(rows / case["new"], 131072, 262144 * 8 / (kv_heads * case["seqs"]))
        case["context"] = max(0, int(tokens) - case["new"])
    else:
        case.update(dtype=rng.choice(["f16", "f16", "f32"]), seqs=_log_uniform(rng, 1, 64), context=_log_uniform(rng, 1, 131072))
    if op in ("chunk", "window") and (op == "window" or rng.random() < 0.4):
        case["window"] = _log_uniform(rng, 1, max(1, min(8192, 1200000 // (case["seqs"] * kv_heads))))
        case["sinks"] = rng.choice([0, 1, 4, 4, 16, 130])
    if case["seqs"] > 1 and rng.random() < 0.7:
        case["min_context"] = case["context"] // rng.choice([2, 8, 1000])
        case["min_new"] = max(0 if op == "window" else 1, case["new"] // rng.choice([1, 2, 8, 1000]))
    else:
        case.update(min_context=case["context"], min_new=case["new"])
    if op == "window":
        case["min_context"] = max(1, case["min_context"])
    return case


def _lengths(case):
    """Tokens of every sequence before the call, and new ones: properties of the case, the same for every seed."""
    rng = random.Random(case["context"] * 1009 + case["seqs"])
    return ([rng.randint(case["min_context"], case["context"]) for _ in range(case["seqs"])],
            [rng.randint(case["min_new"], case["new"]) for _ in range(case["seqs"])])


def _pages_up(tokens):
    return (tokens + GROUP - 1) // GROUP


def _hidden(case, first):
    """Tokens [from, to) that no query from position `first` on sees."""
    return (case["sinks"], max(case["sinks"], first + 1 - case["window"])) if case["window"] else (0, 0)


# ---- inputs: keys with outlier channels under RoPE, quantized and packed with plain torch -----


def _generator(seed, stream):
    g = torch.Generator(device=DEVICE)
    g.manual_seed((seed * 1000003 + stream) % (2 ** 63))
    return g


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _keys(case, seed, generator, positions):
    """Post-RoPE keys [..., kv_heads, d] of the given positions: N(0, 1) with 2 outlier channels of 8 times the size per head."""
    heads = case["kv_heads"]
    k = torch.randn((*positions.shape, heads, HEAD_DIM), generator=generator, device=DEVICE)
    channel_rng = random.Random(seed)
    size = torch.ones((heads, HEAD_DIM))
    for h in range(heads):
        for pair in channel_rng.sample(range(PAIRS), 2):
            size[h, pair + PAIRS * channel_rng.randrange(2)] = 8.0
    k *= size.to(DEVICE)
    freq = 5.0e5 ** (-torch.arange(PAIRS, device=DEVICE, dtype=torch.float64) / PAIRS)
    angle = positions.double()[..., None, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    x, y = k[..., :PAIRS], k[..., PAIRS:]
    return torch.cat([x * cos - y * sin, y * cos + x * sin], dim=-1).to(torch.float16 if case["dtype"] == "f16" else torch.float32)


def _half(x):
    """float64 -> fp16 in one rounding: by way of fp32 rounded to odd."""
    f = x.float()
    f = torch.where(f.double().abs() > x.abs(), torch.nextafter(f, torch.zeros_like(f)), f)
    inexact = (f.double() != x).int()
    return (f.contiguous().view(torch.int32) | inexact).view(torch.float32).half()


def _quantize_keys(case, keys, valid):
    """keys [pages, 128, heads, d], valid [pages, 128]: angle and radius codes [pages, 128, heads, 64], fp16 parameters
    [pages, heads, 64]: (scale, zero) of the radius and, with grouped angles, of the angle."""
    x, y = keys[..., :PAIRS].float(), keys[..., PAIRS:].float()
    rho = torch.sqrt(x * x + y * y)
    theta = torch.atan2(y.double(), x.double())
    there = valid[:, :, None, None]
    r_levels, t_levels = 2 ** case["r_bits"], 2 ** case["t_bits"]
    z = rho.masked_fill(~there, math.inf).amin(dim=1)
    s = ((rho.masked_fill(~there, -math.inf).amax(dim=1) - z) / r_levels).half()
    z = z.half()
    c = torch.floor((rho - z.float()[:, None]) / s.float()[:, None]).nan_to_num(0.0).clamp_(0, r_levels - 1)
    params = [s, z]
    if case["grouped_angles"]:
        tz = theta.masked_fill(~there, math.inf).amin(dim=1)
        ts = _half((theta.masked_fill(~there, -math.inf).amax(dim=1) - tz) / t_levels)
        tz = _half(tz)
        a = torch.floor((theta - tz.double()[:, None]) / ts.double()[:, None]).nan_to_num(0.0)
        params += [ts, tz]
    else:
        # a pair on an axis or a diagonal sits exactly on an edge and belongs to the upper bin
        a = torch.floor((theta + math.pi) * (t_levels / (2 * math.pi)) + 1e-9)
    a = a.clamp_(0, t_levels - 1)
    return (a * there).to(torch.uint8), (c * there).to(torch.uint8), params


def _pack_keys(case, a, c, params):
    """The pools' layout: codes [pages, heads, 4 blocks, 128 tokens, 16 symbols], params {s, z} per pair."""
    n, _, heads, _ = a.shape
    symbol = ((a << case["r_bits"]) | c).view(n, GROUP, heads, 4, 16).permute(0, 2, 3, 1, 4)
    if case["r_bits"] + case["t_bits"] == 6:
        four = symbol.reshape(n, heads, 4, GROUP, 4, 4).to(torch.int32)
        word = four[..., 0] | (four[..., 1] << 6) | (four[..., 2] << 12) | (four[..., 3] << 18)
        symbol = torch.stack([word & 255, (word >> 8) & 255, word >> 16], dim=-1).to(torch.uint8).flatten(-2)
    pairs = [torch.stack(two, dim=-1) for two in zip(params[::2], params[1::2])]
    return symbol.contiguous(), (torch.stack(pairs, dim=2) if len(pairs) == 2 else pairs[0]).contiguous()


def _quantize_values(case, v):
    """Token-wise codes [..., d] and fp16 (scale, zero) [...] of values [..., d]."""
    v = v.float()
    levels = 2 ** case["v_bits"] - 1
    low, high = v.amin(dim=-1), v.amax(dim=-1)
    s, z = ((high - low) / levels).half(), low.half()
    code = torch.round((v - z.float()[..., None]) / s.float()[..., None]).nan_to_num(0.0).clamp_(0, levels)
    return code.to(torch.int32), s, z


def _value_halves(case, code):
    """The 16-bit halves that codes [..., d] fill in their units: [..., 16 slices, halves of 16 / bits dims]."""
    b = case["v_bits"]
    per_half = 4 if b == 4 else 8
    field = code.view(*code.shape[:-1], 16, 8 // per_half, per_half) << (b * torch.arange(per_half, device=DEVICE, dtype=torch.int32))
    bits = field.sum(dim=-1, dtype=torch.int32)
    return torch.where(bits >= 32768, bits - 65536, bits).to(torch.int16)


def _file_values(case, state, values, page, offset):
    """Values [n, heads, d] into the pool at the n places (page, offset)."""
    if case["v_bits"] == 16:
        state["v_pool"].permute(0, 2, 1, 3)[page, offset] = values
        return
    tokens = 16 // case["v_bits"]
    code, s, z = _quantize_values(case, values)
    halves = _value_halves(case, code)                                   # [n, heads, 16, 2 or 1]
    # a unit: [token pair, part of the slice's dims, token of the pair]
    parts = halves.shape[-1]
    pool = state["v_pool"].view(torch.int16).view(-1, case["kv_heads"], GROUP // tokens, 16, tokens // 2, parts, 2).permute(0, 2, 4, 6, 1, 3, 5)
    pool[page, offset // tokens, offset % tokens // 2, offset % 2] = halves
    state["v_params"].permute(0, 2, 1, 3)[page, offset] = torch.stack([s, z], dim=-1)


def _pools(case, total):
    """Zeroed pools of `total` pages."""
    heads, unit = case["kv_heads"], 2 * (case["r_bits"] + case["t_bits"])
    sets = (2,) if case["grouped_angles"] else ()
    state = dict(codes=torch.zeros((total, heads, 4, GROUP, unit), dtype=torch.uint8, device=DEVICE),
                 params=torch.zeros((total, heads, *sets, PAIRS, 2), dtype=torch.float16, device=DEVICE), v_params=None)
    if case["v_bits"] == 16:
        state["v_pool"] = torch.zeros((total, heads, GROUP, HEAD_DIM), dtype=torch.float16, device=DEVICE)
    else:
        tokens = 16 // case["v_bits"]
        state["v_pool"] = torch.zeros((total, heads, GROUP // tokens, 16, 16), dtype=torch.uint8, device=DEVICE)
        state["v_params"] = torch.zeros((total, heads, GROUP, 2), dtype=torch.float16, device=DEVICE)
    return state


SLICE = 256                    # pages of the cache that are made at a time


def _cached_pages(case):
    """(sequence, page of it) of the pages that an attention call reads, sequence by sequence."""
    before, new = _lengths(case)
    found = []
    for s in range(case["seqs"]):
        total = before[s] + new[s]
        first = before[s] if case["op"] == "chunk" else total - 1
        low, high = _hidden(case, first)
        found += [(s, p) for p in range(_pages_up(total)) if p < _pages_up(low) or p >= high // GROUP]
    return found


def _contents(case, seed, pages):
    """What the pages hold, SLICE of them at a time: (first, keys, values, valid) -- [pages, 128, heads, d] and [pages, 128]."""
    before, new = _lengths(case)
    generator = _generator(seed, 1)
    length = _ints([before[s] + new[s] for s, _ in pages])
    index = _ints([p for _, p in pages])
    for at in range(0, len(pages), SLICE):
        positions = index[at:at + SLICE, None] * GROUP + torch.arange(GROUP, device=DEVICE)
        keys = _keys(case, seed, generator, positions)
        values = torch.randn(keys.shape, generator=generator, device=DEVICE).half()
        yield at, keys, values, positions < length[at:at + SLICE, None]


def _queries(case, seed, rows):
    q = torch.randn((rows, case["q_heads"], HEAD_DIM), generator=_generator(seed, 3), device=DEVICE)
    return q.to(torch.float16 if case["dtype"] == "f16" else torch.float32)


def _in_tail(case, length, page):
    return case["tail"] and length % GROUP != 0 and page == length // GROUP


def prepare(case, seed):
    before, new = _lengths(case)
    seqs, heads = case["seqs"], case["kv_heads"]
    total_new = sum(new)
    state = dict(case=case, sm_scale=1.0 / math.sqrt(HEAD_DIM), max_seq_len=max(b + n for b, n in zip(before, new)))
    order = torch.Generator().manual_seed(seed)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    width = max(1, _pages_up(state["max_seq_len"]))

    if case["op"] == "plan":
        have = [_pages_up(b) for b in before]
        need = sum(_pages_up(b + n) - h for b, n, h in zip(before, new, have))
        ids = torch.randperm(sum(have) + need + 7, generator=order).to(torch.int32)
        table = torch.full((seqs, width), -1, dtype=torch.int32)
        held = torch.arange(width)[None, :] < torch.tensor(have)[:, None]
        table[held] = ids[:sum(have)]
        n_free = int(need * case["free"]) + (7 if case["free"] == 1.0 else 0)
        state.update(seq_lens=_ints(before), new_lens=_ints(new), free_pages=ids[sum(have):sum(have) + max(1, n_free)].to(DEVICE),
                     block_table=table.to(DEVICE), starts=torch.zeros(seqs + 1, dtype=torch.int32, device=DEVICE),
                     slots=torch.zeros(total_new, dtype=torch.int64, device=DEVICE),
                     lens_after=torch.zeros(seqs, dtype=torch.int32, device=DEVICE),
                     counts=torch.zeros(2, dtype=torch.int32, device=DEVICE))
        return state

    if case["op"] == "append":
        first = [0]
        for b, n in zip(before, new):
            first.append(first[-1] + _pages_up(b + n))
        ids = torch.randperm(first[-1], generator=order).to(torch.int32)
        table = torch.full((seqs, width), -1, dtype=torch.int32)
        for s in range(seqs):
            table[s, :first[s + 1] - first[s]] = ids[first[s]:first[s + 1]]
        state.update(_pools(case, first[-1]))
        seq = torch.repeat_interleave(torch.arange(seqs), torch.tensor(new))
        position = torch.arange(total_new) - torch.tensor(starts)[seq] + torch.tensor(before)[seq]
        slots = table[seq, position // GROUP].long() * GROUP + position % GROUP
        generator = _generator(seed, 1)
        residual = _keys(case, seed, generator, torch.arange(GROUP, device=DEVICE).expand(seqs, GROUP)).half().permute(0, 2, 1, 3)
        keys = _keys(case, seed, generator, position.to(DEVICE))
        state.update(keys=keys, values=torch.randn(keys.shape, generator=generator, device=DEVICE).half(), starts=_ints(starts),
                     seq_lens=_ints(before), slots=slots.to(DEVICE), residual=residual.contiguous(), block_table=table.to(DEVICE),
                     groups=sum((b % GROUP + n) // GROUP for b, n in zip(before, new)))
        return state

    pages = _cached_pages(case)
    ids = torch.randperm(len(pages), generator=order).to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32)
    seq_of, page_of = torch.tensor([s for s, _ in pages]), torch.tensor([p for _, p in pages])
    table[seq_of, page_of] = ids
    state.update(_pools(case, len(pages)))
    state["residual"] = torch.zeros((seqs, heads, GROUP, HEAD_DIM), dtype=torch.float16, device=DEVICE) if case["tail"] else None
    place = torch.arange(GROUP, device=DEVICE)
    for at, keys, values, valid in _contents(case, seed, pages):
        n = keys.shape[0]
        to = ids[at:at + n].long().to(DEVICE)
        state["codes"][to], state["params"][to] = _pack_keys(case, *_quantize_keys(case, keys, valid))
        _file_values(case, state, values.flatten(0, 1), to.repeat_interleave(GROUP), place.repeat(n))
        for i, (s, p) in enumerate(pages[at:at + n]):
            length = before[s] + new[s]
            if _in_tail(case, length, p):
                state["codes"][to[i]] = 0
                state["params"][to[i]] = 0
                state["residual"][s, :, :length % GROUP] = keys[i, :length % GROUP].half().permute(1, 0, 2)
    chunk = case["op"] == "chunk"
    rows = total_new if chunk else seqs
    state.update(q=_queries(case, seed, rows), block_table=table.to(DEVICE),
                 seq_lens=_ints([b + n for b, n in zip(before, new)]),
                 out=torch.zeros((rows, case["q_heads"], HEAD_DIM), dtype=torch.float16 if chunk else torch.float32, device=DEVICE))
    if chunk:
        state.update(starts=_ints(starts), max_new=max(new))
    return state


# ---- one pass --------------------------------------------------------------------------------


def _handles(state):
    """The cache's layout and the call's workspace, which a program makes once for its shapes and keeps."""
    if "layout" not in state:
        import paper_2502_00527_amd as pq
        case = state["case"]
        layout = pq.Layout(HEAD_DIM, case["r_bits"], case["t_bits"], GROUP, case["kv_heads"], int(case["grouped_angles"]))
        state.update(pq=pq, layout=layout)
        size = 0
        if case["op"] == "chunk":
            size = pq.pq_chunk_workspace_bytes(layout, case["seqs"], case["q_heads"], state["q"].shape[0], state["max_seq_len"])
        elif case["op"] == "window":
            size = pq.pq_window_workspace_bytes(layout, case["seqs"], case["q_heads"], state["max_seq_len"], case["window"], case["sinks"])
        state["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEVICE)
    return state["pq"], state["layout"]


def _run_own(state):
    case = state["case"]
    pq, layout = _handles(state)
    if case["op"] == "plan":
        pq.pq_plan_pages(layout, state["seq_lens"], state["new_lens"], state["free_pages"], state["block_table"], state["starts"],
                         state["slots"], state["lens_after"], state["counts"])
        return [state[k] for k in ("block_table", "starts", "slots", "lens_after", "counts")]
    if case["op"] == "append":
        pq.pq_append_chunk(layout, state["keys"], state["values"], state["starts"], state["seq_lens"], state["slots"], state["residual"],
                           state["block_table"], state["codes"], state["params"], state["v_pool"], case["v_bits"], state["v_params"])
        return [state[k] for k in ("residual", "codes", "params", "v_pool", "v_params")]
    if case["op"] == "chunk":
        pq.pq_chunk_attention(layout, state["q"], state["starts"], state["codes"], state["params"], state["v_pool"], state["block_table"],
                              state["seq_lens"], state["max_seq_len"], state["sm_scale"], state["out"], state["workspace"],
                              state["residual"], case["v_bits"], state["v_params"], case["window"], case["sinks"])
    else:
        pq.pq_window_attention(layout, state["q"], state["codes"], state["params"], state["v_pool"], state["block_table"],
                               state["seq_lens"], state["max_seq_len"], case["window"], case["sinks"], state["sm_scale"], state["out"],
                               state["workspace"], state["residual"], case["v_bits"], state["v_params"])
    return state["out"]


def _plan(state):
    """Pages and slots of the new tokens: prefix sums over the sequences, then one place for each token."""
    length, new, free, table = state["seq_lens"].long(), state["new_lens"].long(), state["free_pages"], state["block_table"]
    have, after = (length + GROUP - 1) // GROUP, (length + new + GROUP - 1) // GROUP
    first = torch.cumsum(after - have, 0) - (after - have)
    ends = torch.cumsum(new, 0)
    state["starts"][1:] = ends
    page = torch.arange(table.shape[1], device=DEVICE)[None, :]
    from_free = first[:, None] + page - have[:, None]
    got = torch.where(from_free < free.shape[0], free[from_free.clamp(0, free.shape[0] - 1)], -1)
    table.copy_(torch.where((page >= have[:, None]) & (page < after[:, None]), got, table))
    token = torch.arange(state["slots"].shape[0], device=DEVICE)
    seq = torch.searchsorted(ends, token, right=True)
    position = length[seq] + token - (ends - new)[seq]
    at = table[seq, position // GROUP].long()
    state["slots"].copy_(torch.where(at >= 0, at * GROUP + position % GROUP, -1))
    state["lens_after"].copy_(length + new)
    state["counts"].copy_(torch.stack([(after - have).sum(), new.sum()]))
    return [state[k] for k in ("block_table", "starts", "slots", "lens_after", "counts")]


def _append(state):
    """Complete groups from the residual's rows and the new keys are quantized and packed, the rest stays as fp16 rows; value rows
    go to their slots."""
    case, starts, length, residual = state["case"], state["starts"].long(), state["seq_lens"].long(), state["residual"]
    seqs, heads = case["seqs"], case["kv_heads"]
    new = starts[1:] - starts[:-1]
    held = length % GROUP
    complete = (held + new) // GROUP
    keys = state["keys"].half()
    rows = torch.cat([residual.permute(0, 2, 1, 3).reshape(seqs * GROUP, heads, HEAD_DIM), keys])
    place = torch.arange(GROUP, device=DEVICE)
    if state["groups"]:
        seq = torch.repeat_interleave(torch.arange(seqs, device=DEVICE), complete, output_size=state["groups"])
        group = torch.arange(state["groups"], device=DEVICE) - (torch.cumsum(complete, 0) - complete)[seq]
        within = group[:, None] * GROUP + place
        source = torch.where(within < held[seq, None], seq[:, None] * GROUP + within,
                             seqs * GROUP + (starts[seq] - held[seq])[:, None] + within)
        taken = rows[source.flatten()].view(-1, GROUP, heads, HEAD_DIM)
        page = state["block_table"][seq, length[seq] // GROUP + group].long()
        state["codes"][page], state["params"][page] = _pack_keys(case, *_quantize_keys(case, taken, torch.ones_like(within, dtype=torch.bool)))
    # rows of the incomplete group: from the new keys, or as they were
    rest = (held + new) % GROUP
    source = (starts[:-1] - held + complete * GROUP)[:, None] + place
    fresh = (place < rest[:, None]) & ((complete > 0)[:, None] | (place >= held[:, None]))
    moved = keys[source.clamp(0, keys.shape[0] - 1).flatten()].view(seqs, GROUP, heads, HEAD_DIM).permute(0, 2, 1, 3)
    residual.copy_(torch.where(fresh[:, None, :, None], moved, residual))
    _file_values(case, state, state["values"], state["slots"] // GROUP, state["slots"] % GROUP)
    return [state[k] for k in ("residual", "codes", "params", "v_pool", "v_params")]


def _gathered(state, pages, tail):
    """Keys and values in 32 bits of pool pages [seqs, n] (-1: any), tail [seqs, n] where the residual's rows stand for the page's
    keys: [seqs, heads, n * 128, d]."""
    case = state["case"]
    seqs, n = pages.shape
    heads, r, t = case["kv_heads"], case["r_bits"], case["t_bits"]
    at = pages.clamp(min=0).long().flatten()
    code = state["codes"][at]
    if r + t == 6:
        three = code.view(*code.shape[:-1], 4, 3).int()
        word = three[..., 0] | (three[..., 1] << 8) | (three[..., 2] << 16)
        code = ((word[..., None] >> torch.tensor([0, 6, 12, 18], device=DEVICE)) & 63).flatten(-2)
    code = code.permute(0, 1, 3, 2, 4).flatten(-2)                       # [pages, heads, 128, 64]
    params = state["params"][at].float().view(seqs * n, heads, -1, PAIRS, 2)
    rho = ((code & (2 ** r - 1)).float() + 0.5) * params[:, :, 0, None, :, 0] + params[:, :, 0, None, :, 1]
    theta = (code >> r).float() + 0.5
    if case["grouped_angles"]:
        theta = theta * params[:, :, 1, None, :, 0] + params[:, :, 1, None, :, 1]
    else:
        theta = theta * (2 * math.pi / 2 ** t) - math.pi
    k = torch.cat([rho * theta.cos(), rho * theta.sin()], dim=-1).view(seqs, n, heads, GROUP, HEAD_DIM)
    if tail is not None:
        k = torch.where(tail[:, :, None, None, None], state["residual"].float()[:, None], k)
    if case["v_bits"] == 16:
        v = state["v_pool"][at].float()
    else:
        b = case["v_bits"]
        parts, bits = (2, 4) if b == 4 else (1, 8)
        half = state["v_pool"][at].view(torch.int16).int().view(seqs * n, heads, GROUP * b // 16, 16, 8 // b, parts, 2)
        field = (half[..., None] >> (b * torch.arange(bits, device=DEVICE))) & (2 ** b - 1)
        # [block, slice, pair, part, token of the pair, dim] -> token, dim
        field = field.permute(0, 1, 2, 4, 6, 3, 5, 7).reshape(seqs * n, heads, GROUP, HEAD_DIM).float()
        vp = state["v_params"][at].float()
        v = field * vp[..., 0:1] + vp[..., 1:2]
    v = v.view(seqs, n, heads, GROUP, HEAD_DIM)
    return [x.permute(0, 2, 1, 3, 4).reshape(seqs, heads, n * GROUP, HEAD_DIM) for x in (k, v)]


def _visible(case, position, token):
    """Whether a query at `position` sees a token."""
    seen = (token <= position) & (position >= 0)
    return seen & ((token > position - case["window"]) | (token < case["sinks"])) if case["window"] else seen


def _softmax_values(scores, seen, v):
    """softmax over the visible tokens, times the values; rows that see nothing are zero."""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total > 0, total, 1.0)


def _chunk(state):
    case, starts, length, table = state["case"], state["starts"].long(), state["seq_lens"].long(), state["block_table"]
    seqs, heads, n = case["seqs"], case["kv_heads"], state["max_new"]
    group = case["q_heads"] // heads
    new = starts[1:] - starts[:-1]
    pages = torch.arange(table.shape[1], device=DEVICE)
    tail = (pages == (length // GROUP)[:, None]) & (length % GROUP != 0)[:, None] if case["tail"] else None
    k, v = _gathered(state, table, tail)
    i = torch.arange(n, device=DEVICE)
    row = (starts[:-1, None] + i).clamp(max=state["q"].shape[0] - 1)
    q = state["q"][row.flatten()].float().view(seqs, n, heads, group, HEAD_DIM).permute(0, 2, 3, 1, 4).reshape(seqs, heads, group * n, HEAD_DIM)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(state["sm_scale"])
    seen = _visible(case, (length - new)[:, None, None] + i[None, :, None], torch.arange(k.shape[2], device=DEVICE))
    scores = scores.view(seqs, heads, group, n, -1)
    out = _softmax_values(scores, seen[:, None, None], v[:, :, None])
    out = out.permute(0, 3, 1, 2, 4).reshape(seqs * n, case["q_heads"], HEAD_DIM)
    # rows past a sequence's chunk go to a row behind the last one
    rows = state["q"].shape[0]
    to = torch.where(i < new[:, None], starts[:-1, None] + i, rows).flatten()
    whole = torch.empty((rows + 1, case["q_heads"], HEAD_DIM), device=DEVICE)
    whole[to] = out
    state["out"].copy_(whole[:rows])
    return state["out"]


def _window(state):
    case, length, table = state["case"], state["seq_lens"].long(), state["block_table"]
    seqs, heads = case["seqs"], case["kv_heads"]
    # the sinks' pages and the window's, as far as any sequence has them
    sink_pages = _pages_up(case["sinks"])
    begin = torch.clamp((length - case["window"]) // GROUP, min=sink_pages)
    n = min(table.shape[1], sink_pages + _pages_up(case["window"]) + 1)
    i = torch.arange(n, device=DEVICE)
    page = torch.where(i < sink_pages, i, begin[:, None] + i - sink_pages)
    tail = (page == (length // GROUP)[:, None]) & (length % GROUP != 0)[:, None] if case["tail"] else None
    k, v = _gathered(state, torch.gather(table, 1, page.clamp(max=table.shape[1] - 1)), tail)
    token = (page[:, :, None] * GROUP + torch.arange(GROUP, device=DEVICE)).flatten(1)
    q = state["q"].float().view(seqs, heads, -1, HEAD_DIM)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(state["sm_scale"])
    out = _softmax_values(scores, _visible(case, length[:, None] - 1, token)[:, None, None], v)
    state["out"].copy_(out.view(seqs, case["q_heads"], HEAD_DIM))
    return state["out"]


def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plan, "append": _append, "chunk": _chunk, "window": _window}[state["case"]["op"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------


def work(case):
    """Every input read once, every output written once; multiply-adds of q.k and p.v as two operations."""
    before, new = _lengths(case)
    heads, tokens = case["kv_heads"], sum(new)
    code = PAIRS * (case["r_bits"] + case["t_bits"]) / 8 + (4 if case["grouped_angles"] else 2)
    value = 2 * HEAD_DIM if case["v_bits"] == 16 else HEAD_DIM * case["v_bits"] / 8 + 4
    element = 2 if case["dtype"] == "f16" else 4
    row = 2 * HEAD_DIM                                                   # of the residual
    if case["op"] == "plan":
        taken = sum(_pages_up(b + n) - _pages_up(b) for b, n in zip(before, new))
        return dict(bytes=8 * tokens + 8 * taken + 16 * case["seqs"], flops=4 * tokens)
    if case["op"] == "append":
        data = tokens * (heads * (HEAD_DIM * element + 2 * HEAD_DIM + value) + 8)
        for b, n in zip(before, new):
            held = b % GROUP
            done = (held + n) // GROUP * GROUP
            data += heads * (done * code + (held * row if done else 0) + ((held + n - done) if done else n) * row)
        return dict(bytes=data, flops=tokens * heads * (PAIRS * 12 + HEAD_DIM * (0 if case["v_bits"] == 16 else 5)))
    data, scores = 0, 0
    for b, n in zip(before, new):
        total = b + n
        n = n if case["op"] == "chunk" else 1
        low, high = _hidden(case, total - n)
        read = total - max(0, min(high, total) - low)
        in_tail = min(total % GROUP, read) if case["tail"] else 0
        data += heads * (read * (code + value) + in_tail * (row - code))
        window = case["window"] or total
        for p in range(total - n, total):
            scores += min(p + 1, window) + min(case["sinks"], max(0, p + 1 - window))
    rows = tokens if case["op"] == "chunk" else case["seqs"]
    data += rows * case["q_heads"] * HEAD_DIM * (element + (2 if case["op"] == "chunk" else 4))
    return dict(bytes=data, flops=scores * case["q_heads"] * 4 * HEAD_DIM)


# ---- from the definitions, in 64 bits ------------------------------------------------------------


def _exact_append(case, seed):
    state = prepare(case, seed)
    before, new = _lengths(case)
    pools = {k: state[k].double() for k in ("residual", "params", "v_pool", "v_params") if state[k] is not None}
    r, t = case["r_bits"], case["t_bits"]
    table, at = state["block_table"].tolist(), 0
    for s, (b, n) in enumerate(zip(before, new)):
        keys, values = state["keys"][at:at + n], state["values"][at:at + n].double()
        at += n
        rows = torch.cat([state["residual"][s, :, :b % GROUP].permute(1, 0, 2), keys.half()]).double()
        done = rows.shape[0] // GROUP
        for g in range(done):
            group = rows[g * GROUP:(g + 1) * GROUP]
            x, y = group[..., :PAIRS], group[..., PAIRS:]
            found = [torch.hypot(x, y)] + ([torch.atan2(y, x)] if case["grouped_angles"] else [])
            pairs = [torch.stack([(f.amax(0) - f.amin(0)) / 2 ** bits, f.amin(0)], dim=-1) for f, bits in zip(found, (r, t))]
            pools["params"][table[s][b // GROUP + g]] = torch.stack(pairs, dim=1) if len(pairs) == 2 else pairs[0]
        rest = rows[done * GROUP:]
        pools["residual"][s, :, :rest.shape[0]] = rest.permute(1, 0, 2)
        position = torch.arange(b, b + n, device=DEVICE)
        page, offset = state["block_table"][s].long()[position // GROUP], position % GROUP
        if case["v_bits"] == 16:
            pools["v_pool"].transpose(1, 2)[page, offset] = values
        else:
            low, high = values.amin(-1), values.amax(-1)
            pools["v_params"].transpose(1, 2)[page, offset] = torch.stack([(high - low) / (2 ** case["v_bits"] - 1), low], dim=-1)
    return [pools["residual"], None, pools["params"], pools["v_pool"] if case["v_bits"] == 16 else None, pools.get("v_params")]


def exact(case, seed):
    """Parameters, rows and attention outputs in float64; codes and slots are whole numbers and have none."""
    if case["op"] == "plan":
        return None
    if case["op"] == "append":
        return _exact_append(case, seed)
    before, new = _lengths(case)
    heads = case["kv_heads"]
    group = case["q_heads"] // heads
    pages = _cached_pages(case)
    kept = []
    for at, keys, values, valid in _contents(case, seed, pages):
        a, c, params = _quantize_keys(case, keys, valid)
        p = [x.double()[:, None] for x in params]
        radius = (c.double() + 0.5) * p[0] + p[1]
        turn = (a.double() + 0.5) * p[2] + p[3] if case["grouped_angles"] else (a.double() + 0.5) * (math.tau / 2 ** case["t_bits"]) - math.pi
        k = torch.cat([radius * torch.cos(turn), radius * torch.sin(turn)], dim=-1)
        for i, (s, page) in enumerate(pages[at:at + keys.shape[0]]):
            if _in_tail(case, before[s] + new[s], page):
                k[i] = keys[i].half().double()
        v = values.double()
        if case["v_bits"] != 16:
            code, vs, vz = _quantize_values(case, values)
            v = code.double() * vs.double()[..., None] + vz.double()[..., None]
        kept.append((k, v))
    k_all, v_all = (torch.cat(x) for x in zip(*kept))
    chunk = case["op"] == "chunk"
    q_all = _queries(case, seed, sum(new) if chunk else case["seqs"]).double()
    outs, row, at = [], 0, 0
    for s in range(case["seqs"]):
        total = before[s] + new[s]
        n = new[s] if chunk else 1
        mine = [p for owner, p in pages[at:] if owner == s]
        k, v = (x[at:at + len(mine)].flatten(0, 1).permute(1, 0, 2).contiguous() for x in (k_all, v_all))
        at += len(mine)
        token = (_ints(mine)[:, None] * GROUP + torch.arange(GROUP, device=DEVICE)).flatten()
        position = torch.arange(total - n, total, device=DEVICE)[:, None]
        hidden = token > position
        if case["window"]:
            hidden = hidden | ((position - token >= case["window"]) & (token >= case["sinks"]))
        q = q_all[row:row + n].view(n, heads, group, HEAD_DIM)
        row += n
        result = torch.zeros((n, heads, group, HEAD_DIM), dtype=torch.float64, device=DEVICE)
        for h in range(heads):
            for g in range(group):
                weight = torch.softmax((q[:, h, g] @ k[h].t().contiguous() / math.sqrt(HEAD_DIM)).masked_fill(hidden, -math.inf), dim=-1)
                result[:, h, g] = weight @ v[h]
        outs.append(result.view(n, case["q_heads"], HEAD_DIM))
    return torch.cat(outs)
