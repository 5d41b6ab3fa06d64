"""Long caches that a step reads or keeps a part of, as calls that can be timed and checked: bounds of each page's
keys, the choice of pages by a cheap score of each query against them, attention over the chosen pages, attention
that also sums each page's weight, and the eviction of pages by that sum.

A case is one such call.  `run` makes it through the library where `own` is true and computes the same
in elementary torch operations where it is not.  The packed cache is made here with plain torch, from
keys with outlier channels under RoPE.  Bounds, choices and block tables are whole numbers that their definitions fix.

Definitions.  Block b of a head's 128 channels is pairs 16 b .. 16 b + 15, both coordinates: 32 channels.
  bounds   of a complete page and KV head: lo_i, hi_i smallest and largest reconstructed key element of channel i over the page's
           tokens, M_b largest |lo_i|, |hi_i| of a block, scale_b = M_b / 127, and as 8-bit numbers
           c_i = round((lo_i + hi_i) / 2 * (127 / M_b)),  w_i = round((hi_i - lo_i) / 2 * (127 / M_b))   (0 where M_b < 2^-100)
  score    of a page: with m_b = largest |q_i| of the block's channels over the KV head's query heads, q8_i = round(q_i * (127 / m_b)),
           n_b = sum over the block of q8_i c_i + |q8_i| w_i:  (n_0 u_0 + n_1 u_1) + (n_2 u_2 + n_3 u_3), u_b = m_b scale_b, the largest
           of the KV head's query heads: up to rounding 127 times the largest score that a key within the bounds could have
  choice   the first n_first and last n_last pages, and of the others those of the largest scores, n_selected in all; ties: the first ones
  weights  of a page: the sum over its tokens and all query heads of the softmax weights, plus `decay` times what the page had
  eviction of the pages beyond n_kept: those of the smallest weight, but for the first n_first, the last n_last and an incomplete one;
           ties: the first ones
Everything that decides is rounded to 32 bits after each operation, so that whole numbers do not depend on who computes them.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
PAIRS = HEAD_DIM // 2
GROUP = 128                    # tokens of a page
BLOCKS, CHANNELS = 4, 32       # of the bounds
TINY = 2.0 ** -100
DEVICE = "cuda:0"

# ---- cases -----------------------------------------------------------------------------------


def _case(name, op, seqs, kv_heads, context, **more):
    case = dict(name=name, op=op, seqs=seqs, q_heads=4 * kv_heads, kv_heads=kv_heads, context=context, min_context=context,
                new=1, min_new=1, r_bits=4, t_bits=4, grouped_angles=False, v_bits=16, dtype="f16", tail=True, chosen=0, first=0,
                last=1, kept=0, decay=0.0)
    case.update(more)
    return case


def listed():
    return [
        # a decode step of a batch in which some sequences complete a page
        _case("bound_step", "bound", 64, 8, 16384, min_context=200),
        # whole prompts, behind their encoding
        _case("bound_prompts", "bound", 8, 8, 0, new=32768, min_new=20000),
        # one user far into a long document: which of 1024 pages to read
        _case("select_one", "select", 1, 8, 131072, chosen=64, first=1, last=2),
        # a serving batch of ragged lengths, some shorter than what is chosen
        _case("select_batch", "select", 32, 8, 32768, min_context=2000, chosen=32, first=1, last=2),
        # that user's step: latency counts
        _case("sparse_one", "sparse", 1, 8, 131072, chosen=32, first=1, last=2),
        # a batch over long caches
        _case("sparse_batch", "sparse", 16, 8, 32768, chosen=48, first=1, last=4),
        # odd sizes, the paper's own angle quantizer at low bits, quantized values, fp32 queries, seven heads a KV head
        _case("sparse_ragged_v4", "sparse", 13, 4, 20000, q_heads=28, min_context=100, r_bits=3, t_bits=3, grouped_angles=True, v_bits=4,
              dtype="f32", chosen=21, first=0, last=1),
        # one short conversation whose weights are summed
        _case("weights_one", "weights", 1, 8, 3000, decay=1.0),
        # a serving batch at full length: the largest call
        _case("weights_batch", "weights", 16, 8, 32768, decay=0.95),
        # a ragged one, low bits, quantized values
        _case("weights_ragged_v4", "weights", 40, 8, 8000, min_context=300, r_bits=3, t_bits=3, v_bits=4, decay=0.9),
        # between two steps: the sequences of a batch that have begun a page give one back
        _case("evict_step", "evict", 64, 8, 12900, min_context=12700, kept=100, first=1, last=4),
        # long prompts cut down to a quarter
        _case("evict_prompts", "evict", 48, 8, 131072, min_context=40000, kept=256, first=1, last=8),
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


MOST_ROWS = 16 * 8 * 32768     # tokens x KV heads of the largest cache


def draw(rng):
    op = rng.choice(["bound"] * 2 + ["select"] * 3 + ["sparse"] * 4 + ["weights"] * 4 + ["evict"] * 2)
    r_bits, t_bits = rng.choice([(4, 4), (4, 4), (3, 3), (3, 3), (5, 3), (3, 5), (4, 2), (2, 4)])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 32])
    group = rng.choice([1, 2]) if kv_heads == 32 else rng.choice([1, 2, 3, 4, 4, 4, 6, 7, 8, 12, 16])
    case = _case(None, op, 1, kv_heads, 0, q_heads=kv_heads * group, r_bits=r_bits, t_bits=t_bits, grouped_angles=rng.random() < 0.25,
                 v_bits=rng.choice([16, 16, 16, 4, 2]), dtype=rng.choice(["f16", "f16", "f32"]), tail=rng.random() < 0.75)
    del case["name"]
    if op == "evict":
        case["seqs"] = _log_uniform(rng, 1, 200)
        case["context"] = _log_uniform(rng, 1, max(1, min(131072, 48 * 131072 // case["seqs"])))
    elif op == "bound":
        case["seqs"] = _log_uniform(rng, 1, 64)
        case["new"] = _log_uniform(rng, 1, max(1, min(65536, MOST_ROWS // (2 * kv_heads * case["seqs"]))))
        case["context"] = _log_uniform(rng, 1, 16384)
    else:
        # tokens x KV heads x the larger of one and a quarter of the query heads a KV head
        most = MOST_ROWS / max(1.0, group / 4)
        case["seqs"] = _log_uniform(rng, 1, 64)
        case["context"] = _log_uniform(rng, 1, max(1, min(131072, int(most / (kv_heads * case["seqs"])))))
    if case["seqs"] > 1 and rng.random() < 0.7:
        case["min_context"] = max(1, case["context"] // rng.choice([2, 8, 1000]))
        case["min_new"] = max(1, case["new"] // rng.choice([1, 2, 8, 1000]))
    else:
        case.update(min_context=case["context"], min_new=case["new"])
    pages = _pages_up(case["context"])
    if op in ("select", "sparse", "evict"):
        case.update(first=rng.choice([0, 1, 1, 2]), last=rng.choice([1, 1, 2, 4]))
        least = case["first"] + case["last"]
        count = max(least, _log_uniform(rng, 1, max(1, pages)))
        if op == "evict":
            case["kept"] = count
        else:
            case["chosen"] = min(count, max(least, MOST_ROWS // (8 * GROUP * kv_heads * case["seqs"])))
    if op == "weights":
        case["decay"] = rng.choice([0.0, 0.9, 0.99, 1.0])
    return case


def _lengths(case):
    """Tokens of every sequence before the call, and with the new ones: properties of the case, the same for every seed."""
    rng = random.Random(case["context"] * 1009 + case["seqs"])
    before = [rng.randint(case["min_context"], case["context"]) for _ in range(case["seqs"])]
    if case["op"] != "bound":
        return before, before
    if case["new"] == 1:
        before = [b // GROUP * GROUP + GROUP - 1 if s % 8 == 0 else b for s, b in enumerate(before)]     # these complete a page
    return before, [b + rng.randint(case["min_new"], case["new"]) for b in before]


def _pages_up(tokens):
    return (tokens + GROUP - 1) // GROUP


# ---- inputs: keys with outlier channels under RoPE, quantized and packed with plain torch -----


def _generator(seed, stream):
    g = torch.Generator(device=DEVICE)
    g.manual_seed((seed * 1000003 + stream) % (2 ** 63))
    return g


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _keys(case, seed, generator, page):
    """Post-RoPE keys [n, 128, kv_heads, d] of whole pages (numbers in their sequences): what the page is about, plus N(0, 1), with 2 outlier
    channels of 8 times the size per head."""
    heads = case["kv_heads"]
    k = torch.randn((page.shape[0], GROUP, heads, HEAD_DIM), generator=generator, device=DEVICE)
    k += torch.randn((page.shape[0], 1, heads, HEAD_DIM), generator=generator, device=DEVICE)
    channel_rng = random.Random(seed)
    size = torch.ones((heads, HEAD_DIM))
    for h in range(heads):
        for pair in channel_rng.sample(range(PAIRS), 2):
            size[h, pair + PAIRS * channel_rng.randrange(2)] = 8.0
    k *= size.to(DEVICE)
    freq = 5.0e5 ** (-torch.arange(PAIRS, device=DEVICE, dtype=torch.float64) / PAIRS)
    angle = (page[:, None] * GROUP + torch.arange(GROUP, device=DEVICE)).double()[..., None, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    x, y = k[..., :PAIRS], k[..., PAIRS:]
    return torch.cat([x * cos - y * sin, y * cos + x * sin], dim=-1).half()


def _quantize_keys(case, keys, valid):
    """keys [pages, 128, heads, d], valid [pages, 128]: angle and radius codes [pages, 128, heads, 64], fp16 parameters
    [pages, heads, 64]: (scale, zero) of the radius and, with grouped angles, of the angle."""
    x, y = keys[..., :PAIRS].float(), keys[..., PAIRS:].float()
    rho, theta = torch.sqrt(x * x + y * y), torch.atan2(y, x)
    there = valid[:, :, None, None]
    r_levels, t_levels = 2 ** case["r_bits"], 2 ** case["t_bits"]
    z = rho.masked_fill(~there, math.inf).amin(dim=1)
    s = ((rho.masked_fill(~there, -math.inf).amax(dim=1) - z) / r_levels).half()
    z = z.half()
    c = torch.floor((rho - z.float()[:, None]) / s.float()[:, None]).nan_to_num(0.0).clamp_(0, r_levels - 1)
    params = [s, z]
    if case["grouped_angles"]:
        tz = theta.masked_fill(~there, math.inf).amin(dim=1)
        ts = ((theta.masked_fill(~there, -math.inf).amax(dim=1) - tz) / t_levels).half()
        tz = tz.half()
        a = torch.floor((theta - tz.float()[:, None]) / ts.float()[:, None]).nan_to_num(0.0)
        params += [ts, tz]
    else:
        a = torch.floor((theta + math.pi) * (t_levels / (2 * math.pi)))
    a = a.clamp_(0, t_levels - 1)
    return (a * there).to(torch.uint8), (c * there).to(torch.uint8), params


def _pack_keys(case, a, c, params):
    """The pools' layout: codes [pages, heads, 4 blocks, 128 tokens, 16 symbols], params {s, z} per pair."""
    n, _, heads, _ = a.shape
    symbol = ((a << case["r_bits"]) | c).view(n, GROUP, heads, BLOCKS, 16).permute(0, 2, 3, 1, 4)
    if case["r_bits"] + case["t_bits"] == 6:
        four = symbol.reshape(n, heads, BLOCKS, GROUP, 4, 4).to(torch.int32)
        word = four[..., 0] | (four[..., 1] << 6) | (four[..., 2] << 12) | (four[..., 3] << 18)
        symbol = torch.stack([word & 255, (word >> 8) & 255, word >> 16], dim=-1).to(torch.uint8).flatten(-2)
    pairs = [torch.stack(two, dim=-1) for two in zip(params[::2], params[1::2])]
    return symbol.contiguous(), (torch.stack(pairs, dim=2) if len(pairs) == 2 else pairs[0]).contiguous()


def _store_values(case, state, page, values):
    """Values [n, 128, heads, d] into whole pages of the pool."""
    b = case["v_bits"]
    if b == 16:
        state["v_pool"][page] = values.permute(0, 2, 1, 3)
        return
    v = values.float()
    levels = 2 ** b - 1
    low, high = v.amin(dim=-1), v.amax(dim=-1)
    s, z = ((high - low) / levels).half(), low.half()
    code = torch.round((v - z.float()[..., None]) / s.float()[..., None]).nan_to_num(0.0).clamp_(0, levels).to(torch.int32)
    dims = 4 if b == 4 else 8                                            # of a unit's 16-bit half: parts of a slice of 8
    n, _, heads, _ = values.shape
    half = (code.view(n, GROUP, heads, 16, 8 // dims, dims) << (b * torch.arange(dims, device=DEVICE, dtype=torch.int32))).sum(-1, dtype=torch.int32)
    half = torch.where(half >= 32768, half - 65536, half).to(torch.int16)
    # token = block, pair, which of the pair -> [page, head, block, slice, pair, part, which]
    tokens = 16 // b
    half = half.view(n, GROUP // tokens, tokens // 2, 2, heads, 16, 8 // dims).permute(0, 4, 1, 5, 2, 6, 3)
    state["v_pool"][page] = half.contiguous().view(torch.uint8).view(n, heads, GROUP // tokens, 16, 16)
    state["v_params"][page] = torch.stack([s, z], dim=-1).permute(0, 2, 1, 3)


SLICE = 256                    # pages that are made at a time


def _made_pages(case):
    """(sequence, page of it) of the pages that the call deals with, sequence by sequence."""
    before, after = _lengths(case)
    if case["op"] == "bound":
        return [(s, p) for s in range(case["seqs"]) for p in range(before[s] // GROUP, after[s] // GROUP)]
    return [(s, p) for s in range(case["seqs"]) for p in range(_pages_up(after[s]))]


def _weights(case, seed, width):
    """Sums of weights as steps leave them: a few pages have most, some nothing at all."""
    g = _generator(seed, 5)
    w = torch.exp(3.0 * torch.randn((case["seqs"], width), generator=g, device=DEVICE))
    return torch.where(torch.rand(w.shape, generator=g, device=DEVICE) < 0.2, 0.0, w)


def prepare(case, seed):
    before, after = _lengths(case)
    seqs, heads, op = case["seqs"], case["kv_heads"], case["op"]
    width = max(1, _pages_up(max(after)))
    state = dict(case=case, sm_scale=1.0 / math.sqrt(HEAD_DIM), max_seq_len=max(1, max(after)), max_new=max(a - b for a, b in zip(after, before)),
                 lens_before=_ints(before), seq_lens=_ints(after))
    order = torch.Generator().manual_seed(seed)
    if op == "evict":
        pages = [_pages_up(n) for n in after]
        ids = torch.randperm(sum(pages), generator=order).to(torch.int32)
        table = torch.full((seqs, width), -1, dtype=torch.int32)
        table[torch.arange(width) < torch.tensor(pages)[:, None]] = ids
        state.update(block_table=table.to(DEVICE), weights=_weights(case, seed, width),
                     table_after=torch.full((seqs, width), -1, dtype=torch.int32, device=DEVICE),
                     weights_after=torch.zeros((seqs, width), device=DEVICE), lens_after=torch.zeros(seqs, dtype=torch.int32, device=DEVICE),
                     freed=torch.full((sum(pages),), -1, dtype=torch.int32, device=DEVICE), counts=torch.zeros(1, dtype=torch.int32, device=DEVICE))
        return state

    made = _made_pages(case)
    total = len(made) + 3
    ids = torch.randperm(total, generator=order).to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32)
    if op == "bound":
        table = ids[torch.randint(total, (seqs, width), generator=order)]
    table[torch.tensor([s for s, _ in made], dtype=torch.long), torch.tensor([p for _, p in made], dtype=torch.long)] = ids[:len(made)]
    sets = (2,) if case["grouped_angles"] else ()
    state.update(codes=torch.zeros((total, heads, BLOCKS, GROUP, 2 * (case["r_bits"] + case["t_bits"])), dtype=torch.uint8, device=DEVICE),
                 params=torch.zeros((total, heads, *sets, PAIRS, 2), dtype=torch.float16, device=DEVICE),
                 bounds=torch.zeros((total, heads, BLOCKS, 2, CHANNELS), dtype=torch.int8, device=DEVICE),
                 bound_scales=torch.zeros((total, heads, BLOCKS), device=DEVICE), block_table=table.to(DEVICE), v_params=None, residual=None)
    attends = op in ("sparse", "weights")
    if attends and case["v_bits"] == 16:
        state["v_pool"] = torch.zeros((total, heads, GROUP, HEAD_DIM), dtype=torch.float16, device=DEVICE)
    elif attends:
        state["v_pool"] = torch.zeros((total, heads, GROUP * case["v_bits"] // 16, 16, 16), dtype=torch.uint8, device=DEVICE)
        state["v_params"] = torch.zeros((total, heads, GROUP, 2), dtype=torch.float16, device=DEVICE)
    if attends and case["tail"]:
        state["residual"] = torch.zeros((seqs, heads, GROUP, HEAD_DIM), dtype=torch.float16, device=DEVICE)
    length, number = _ints([after[s] for s, _ in made]), _ints([p for _, p in made])
    generator = _generator(seed, 1)
    for at in range(0, len(made), SLICE):
        there = slice(at, at + SLICE)
        keys = _keys(case, seed, generator, number[there])
        to = ids[:len(made)][there].long().to(DEVICE)
        valid = number[there, None] * GROUP + torch.arange(GROUP, device=DEVICE) < length[there, None]
        state["codes"][to], state["params"][to] = _pack_keys(case, *_quantize_keys(case, keys, valid))
        if attends:
            _store_values(case, state, to, torch.randn(keys.shape, generator=generator, device=DEVICE).half())
        if state["residual"] is not None:
            for i, (s, p) in enumerate(made[there]):
                if after[s] % GROUP and p == after[s] // GROUP:                     # the keys of an incomplete page are rows of the residual
                    state["codes"][to[i]] = 0
                    state["params"][to[i]] = 0
                    state["residual"][s, :, :after[s] % GROUP] = keys[i, :after[s] % GROUP].permute(1, 0, 2)
        if op in ("select", "sparse"):
            state["bounds"][to], state["bound_scales"][to] = _bounds_of(case, state["codes"][to], state["params"][to])
    if op == "bound":
        state["groups"] = len(made)
        return state
    q = torch.randn((seqs, case["q_heads"], HEAD_DIM), generator=_generator(seed, 3), device=DEVICE)
    state["q"] = q.to(torch.float16 if case["dtype"] == "f16" else torch.float32)
    if attends:
        state["out"] = torch.zeros((seqs, case["q_heads"], HEAD_DIM), device=DEVICE)
    if op == "weights":
        state.update(weights_before=_weights(case, seed, width), weights=torch.zeros((seqs, width), device=DEVICE))
    else:
        state.update(selected=torch.full((seqs, heads, case["chosen"]), -1, dtype=torch.int32, device=DEVICE),
                     selected_lens=torch.zeros((seqs, heads), dtype=torch.int32, device=DEVICE))
    return state


# ---- one pass --------------------------------------------------------------------------------


def _handles(state):
    """The cache's layout and the call's workspace, which a program makes once for its shapes and keeps."""
    if "layout" not in state:
        import paper_2502_00527_amd as pq
        case = state["case"]
        layout = pq.Layout(HEAD_DIM, case["r_bits"], case["t_bits"], GROUP, case["kv_heads"], int(case["grouped_angles"]))
        state.update(pq=pq, layout=layout)
        seqs, most = case["seqs"], state["max_seq_len"]
        size = 0
        if case["op"] == "select":
            size = pq.pq_select_workspace_bytes(layout, seqs, most)
        elif case["op"] == "sparse":
            size = pq.pq_sparse_workspace_bytes(layout, seqs, case["q_heads"], most, case["chosen"])
        elif case["op"] == "weights":
            size = pq.pq_weights_workspace_bytes(layout, seqs, case["q_heads"], most)
        state["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEVICE)
    return state["pq"], state["layout"]


def _run_own(state):
    case = state["case"]
    pq, layout = _handles(state)
    if case["op"] == "bound":
        pq.pq_bound_pages(layout, state["codes"], state["params"], state["block_table"], state["lens_before"], state["seq_lens"],
                          state["max_new"], state["bounds"], state["bound_scales"])
        return [state["bounds"], state["bound_scales"]]
    if case["op"] == "select":
        pq.pq_select_pages(layout, state["q"], state["bounds"], state["bound_scales"], state["block_table"], state["seq_lens"],
                           state["max_seq_len"], case["first"], case["last"], state["selected"], state["selected_lens"], state["workspace"])
        return [state["selected"], state["selected_lens"]]
    if case["op"] == "sparse":
        pq.pq_sparse_attention(layout, state["q"], state["codes"], state["params"], state["v_pool"], state["bounds"], state["bound_scales"],
                               state["block_table"], state["seq_lens"], state["max_seq_len"], case["first"], case["last"], state["sm_scale"],
                               state["selected"], state["selected_lens"], state["out"], state["workspace"], state["residual"],
                               case["v_bits"], state["v_params"])
        return [state["out"], state["selected"], state["selected_lens"]]
    if case["op"] == "weights":
        pq.pq_decode_attention_weights(layout, state["q"], state["codes"], state["params"], state["v_pool"], state["block_table"],
                                       state["seq_lens"], state["max_seq_len"], state["sm_scale"], state["out"], state["weights"],
                                       state["workspace"], state["weights_before"], case["decay"], state["residual"], case["v_bits"],
                                       state["v_params"])
        return [state["out"], state["weights"]]
    pq.pq_evict_pages(layout, state["block_table"], state["seq_lens"], state["weights"], case["kept"], case["first"], case["last"],
                      state["table_after"], state["lens_after"], state["weights_after"], state["freed"], state["counts"])
    return [state[k] for k in ("table_after", "lens_after", "weights_after", "freed", "counts")]


def _unpack(case, code):
    """Symbols [..., 64 pairs] in token order of codes [..., 4, 128, unit]: [..., 128, 64]."""
    if case["r_bits"] + case["t_bits"] == 6:
        three = code.view(*code.shape[:-1], 4, 3).int()
        word = three[..., 0] | (three[..., 1] << 8) | (three[..., 2] << 16)
        code = ((word[..., None] >> torch.tensor([0, 6, 12, 18], device=DEVICE)) & 63).flatten(-2)
    return code.transpose(-3, -2).flatten(-2)


def _reconstruct(case, code, params):
    """Key elements (x, y), 32 bits, of codes [n, heads, 4, 128, unit]: [n, heads, 128, 64] each.  Angles in 64 bits, rounded once."""
    r, t = case["r_bits"], case["t_bits"]
    symbol = _unpack(case, code)
    params = params.view(*params.shape[:2], -1, 1, PAIRS, 2)
    radius = ((symbol & (2 ** r - 1)).float() + 0.5) * params[:, :, 0, ..., 0].float() + params[:, :, 0, ..., 1].float()
    bins = torch.arange(2 ** t, device=DEVICE, dtype=torch.float64) + 0.5
    angle = (symbol >> r).long()
    if case["grouped_angles"]:
        theta = bins[:, None] * params[:, :, 1, ..., 0].double() + params[:, :, 1, ..., 1].double()     # [n, heads, 2^t, 64]
        cos, sin = (torch.gather(f.float(), 2, angle) for f in (theta.cos(), theta.sin()))
    else:
        theta = bins * (2 * math.pi / 2 ** t) - math.pi
        cos, sin = theta.cos().float()[angle], theta.sin().float()[angle]
    return radius * cos, radius * sin


def _over(number, largest):
    """number / largest with one rounding to 32 bits, 0 where the largest is next to nothing."""
    return torch.where(largest >= TINY, (number / largest.double()).float(), 0.0)


def _bounds_of(case, code, params):
    """Bounds [n, heads, 4, 2, 32] in 8 bits and their scales [n, heads, 4] of whole pages."""
    elements = torch.stack(_reconstruct(case, code, params), dim=-2)                          # [n, heads, 128, 2, 64]
    n, heads = code.shape[:2]
    low, high = (f.view(n, heads, 2, BLOCKS, 16).transpose(2, 3).flatten(-2) for f in (elements.amin(dim=2), elements.amax(dim=2)))
    largest = torch.maximum(low.abs(), high.abs()).amax(dim=-1)
    up = _over(127.0, largest)[..., None]
    centre, half = (low + high) * 0.5 * up, (high - low) * 0.5 * up
    return torch.stack([torch.round(centre), torch.round(half)], dim=-2).to(torch.int8), (largest.double() / 127.0).float()


def _bound(state):
    """Pages that the new tokens complete, found from the lengths, and their bounds."""
    if state["groups"]:
        first, last = state["lens_before"].long() // GROUP, state["seq_lens"].long() // GROUP
        count = last - first
        seq = torch.repeat_interleave(torch.arange(count.shape[0], device=DEVICE), count, output_size=state["groups"])
        page = first[seq] + torch.arange(state["groups"], device=DEVICE) - (torch.cumsum(count, 0) - count)[seq]
        at = state["block_table"][seq, page].long()
        state["bounds"][at], state["bound_scales"][at] = _bounds_of(state["case"], state["codes"][at], state["params"][at])
    return [state["bounds"], state["bound_scales"]]


def _select(state):
    """Pages [seqs, heads, chosen] that each KV head reads, in order; -1 behind them."""
    case, table = state["case"], state["block_table"]
    seqs, heads, chosen = case["seqs"], case["kv_heads"], case["chosen"]
    width = table.shape[1]
    q = state["q"].float().view(seqs, heads, -1, 2, BLOCKS, 16).transpose(3, 4).flatten(-2)        # [seqs, heads, group, 4, 32]
    largest = q.abs().amax(dim=(2, 4))
    q8 = torch.round(q * _over(127.0, largest)[:, :, None, :, None]).permute(0, 1, 3, 2, 4)
    at = table.clamp(min=0).long()
    bound = state["bounds"][at].float().permute(0, 2, 3, 4, 5, 1).contiguous()                      # [seqs, heads, 4, 2, 32, pages]
    number = torch.matmul(q8, bound[:, :, :, 0]) + torch.matmul(q8.abs(), bound[:, :, :, 1])        # whole numbers below 2^24
    term = number * (largest[..., None] * state["bound_scales"][at].permute(0, 2, 3, 1))[:, :, :, None]
    score = ((term[:, :, 0] + term[:, :, 1]) + (term[:, :, 2] + term[:, :, 3])).amax(dim=2)
    page = torch.arange(width, device=DEVICE)
    pages = ((state["seq_lens"].long() + GROUP - 1) // GROUP)[:, None, None]
    sure = (page < case["first"]) | (page >= pages - case["last"])
    rank = torch.where(page >= pages, 2, torch.where(sure, 0, 1)).expand(seqs, heads, width)
    by_score = torch.sort(score, dim=-1, descending=True, stable=True).indices
    by_rank = torch.sort(torch.gather(rank, 2, by_score), dim=-1, stable=True).indices
    count = pages.clamp(max=chosen).expand(seqs, heads, 1)
    place = torch.arange(min(chosen, width), device=DEVICE)
    taken = torch.where(place < count, torch.gather(by_score, 2, by_rank)[..., :place.shape[0]], width).sort(dim=-1).values
    return taken, count[..., 0], at


def _selected(state):
    case = state["case"]
    taken, count, at = _select(state)
    head = torch.arange(case["kv_heads"], device=DEVICE)[None, :, None]
    there = torch.arange(taken.shape[-1], device=DEVICE) < count[..., None]
    row = torch.gather(at[:, None].expand(-1, case["kv_heads"], -1), 2, taken.clamp(max=at.shape[1] - 1)) * case["kv_heads"] + head
    state["selected"][..., :taken.shape[-1]] = torch.where(there, row, -1).int()
    length = state["seq_lens"].long()[:, None]
    state["selected_lens"].copy_((length - ((length + GROUP - 1) // GROUP - count) * GROUP).clamp(min=0))
    return row.clamp(min=0), [state["selected"], state["selected_lens"]]


def _attend(state, row, lens, tail):
    """Attention of one query a sequence over rows [seqs, heads, n] of the pools taken head by head: outputs, and the softmax weights
    [seqs, heads, group, n, 128].  lens [seqs, heads]: tokens in them; tail [seqs, heads]: the page whose keys the residual holds, or -1."""
    case = state["case"]
    seqs, heads, n = row.shape
    at = row.flatten()
    x, y = _reconstruct(case, state["codes"].flatten(0, 1)[at][:, None], state["params"].flatten(0, 1)[at][:, None])
    k = torch.cat([x, y], dim=-1).view(seqs, heads, n, GROUP, HEAD_DIM)
    if state["residual"] is not None:
        here = torch.arange(n, device=DEVICE) == tail[..., None]
        k = torch.where(here[..., None, None], state["residual"].float()[:, :, None], k)
    if case["v_bits"] == 16:
        v = state["v_pool"].flatten(0, 1)[at].float()
    else:
        b = case["v_bits"]
        dims = 4 if b == 4 else 8
        half = state["v_pool"].flatten(0, 1)[at].view(torch.int16).int().view(-1, GROUP * b // 16, 16, 8 // b, 8 // dims, 2)
        field = (half[..., None] >> (b * torch.arange(dims, device=DEVICE))) & (2 ** b - 1)
        # [block, slice, pair, part, which of the pair, dim] -> token, dim
        field = field.permute(0, 1, 3, 5, 2, 4, 6).reshape(-1, GROUP, HEAD_DIM).float()
        vp = state["v_params"].flatten(0, 1)[at].float()
        v = field * vp[..., 0:1] + vp[..., 1:2]
    k, v = k.view(seqs, heads, n * GROUP, HEAD_DIM), v.view(seqs, heads, n * GROUP, HEAD_DIM)
    q = state["q"].float().view(seqs, heads, -1, HEAD_DIM)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(state["sm_scale"])
    scores.masked_fill_(torch.arange(n * GROUP, device=DEVICE) >= lens[:, :, None, None], -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    return torch.matmul(p, v).view(seqs, case["q_heads"], HEAD_DIM), p.view(seqs, heads, -1, n, GROUP)


def _sparse(state):
    row, chosen = _selected(state)
    lens = state["selected_lens"].long()
    tail = torch.where(lens % GROUP != 0, lens // GROUP, -1)
    state["out"].copy_(_attend(state, row, lens, tail)[0])
    return [state["out"], *chosen]


def _summed(state):
    case, length = state["case"], state["seq_lens"].long()
    heads = case["kv_heads"]
    row = state["block_table"].clamp(min=0).long()[:, None] * heads + torch.arange(heads, device=DEVICE)[None, :, None]
    lens = length[:, None].expand(-1, heads)
    out, p = _attend(state, row, lens, torch.where(lens % GROUP != 0, lens // GROUP, -1))
    state["out"].copy_(out)
    there = torch.arange(row.shape[-1], device=DEVICE) < ((length + GROUP - 1) // GROUP)[:, None]
    state["weights"].copy_(torch.where(there, p.sum(dim=-1).sum(dim=(1, 2)) + case["decay"] * state["weights_before"], state["weights"]))
    return [state["out"], state["weights"]]


def _evict(state):
    """The pages of the smallest weights out of the block table, the others moved together."""
    case, table, length = state["case"], state["block_table"], state["seq_lens"].long()[:, None]
    width = table.shape[1]
    page = torch.arange(width, device=DEVICE)
    pages = (length + GROUP - 1) // GROUP
    last = torch.where(length % GROUP != 0, max(1, case["last"]), case["last"])
    sure = (page < case["first"]) | (page >= pages - last)
    held = torch.minimum(pages, case["first"] + last)
    gone = (pages - torch.clamp(held, min=case["kept"])).clamp(min=0)
    by_weight = torch.sort(state["weights"], dim=-1, stable=True).indices
    order = torch.gather(by_weight, 1, torch.sort(torch.gather(sure.int(), 1, by_weight), dim=-1, stable=True).indices)
    evicted = torch.zeros_like(table, dtype=torch.bool).scatter_(1, order, page < gone)
    place = torch.sort(torch.where(evicted, page + width, page), dim=-1).indices
    kept = page < pages - gone
    left = page >= pages
    state["table_after"].copy_(torch.where(left, state["table_after"], torch.where(kept, torch.gather(table, 1, place), -1)))
    state["weights_after"].copy_(torch.where(left, state["weights_after"], torch.where(kept, torch.gather(state["weights"], 1, place), 0.0)))
    state["lens_after"].copy_((length - gone * GROUP)[:, 0])
    state["freed"][:int(gone.sum())] = table[evicted]
    state["counts"].copy_(gone.sum())
    return [state[k] for k in ("table_after", "lens_after", "weights_after", "freed", "counts")]


def run(state):
    if own:
        return _run_own(state)
    if state["case"]["op"] == "select":
        return _selected(state)[1]
    return {"bound": _bound, "sparse": _sparse, "weights": _summed, "evict": _evict}[state["case"]["op"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------


def work(case):
    """Every input read once, every output written once; multiply-adds as two operations."""
    before, after = _lengths(case)
    seqs, heads, queries = case["seqs"], case["kv_heads"], case["q_heads"]
    code = GROUP * PAIRS * (case["r_bits"] + case["t_bits"]) // 8 + PAIRS * (8 if case["grouped_angles"] else 4)   # of a page and head
    value = GROUP * (2 * HEAD_DIM if case["v_bits"] == 16 else HEAD_DIM * case["v_bits"] // 8 + 4)
    bound = 2 * BLOCKS * CHANNELS + 4 * BLOCKS
    query = queries * HEAD_DIM * (2 if case["dtype"] == "f16" else 4)
    pages = [_pages_up(n) for n in after]
    if case["op"] == "bound":
        done = sum(a // GROUP - b // GROUP for a, b in zip(after, before))
        return dict(bytes=done * (4 + heads * (code + bound)) + 8 * seqs, flops=done * heads * GROUP * PAIRS * 9)
    if case["op"] == "evict":
        freed = sum(max(0, p - max(case["kept"], min(p, case["first"] + case["last"]))) for p in pages)
        return dict(bytes=16 * sum(pages) + 4 * freed + 8 * seqs, flops=4 * sum(pages))
    scored = sum(p for p in pages if p > case["chosen"])
    choose = dict(bytes=seqs * (query + 4) + scored * (4 + heads * bound) + heads * (4 * seqs + 4 * sum(min(p, case["chosen"]) for p in pages)),
                  flops=scored * queries * 4 * BLOCKS * CHANNELS)
    if case["op"] == "select":
        return choose
    data, tokens = 0, 0
    for n, p in zip(after, pages):
        n -= max(0, p - case["chosen"]) * GROUP if case["op"] == "sparse" else 0
        rest = n % GROUP if case["tail"] else 0
        data += heads * ((code + value) * (n - rest) / GROUP + rest * (2 * HEAD_DIM + value / GROUP))
        tokens += n
    data += seqs * (query + 4 * queries * HEAD_DIM)
    flops = tokens * queries * 4 * HEAD_DIM
    if case["op"] == "sparse":
        return dict(bytes=data + choose["bytes"] - seqs * query, flops=flops + choose["flops"])
    return dict(bytes=data + sum(pages) * (8 + 4 * (case["decay"] != 0)) + 4 * seqs, flops=flops + tokens * queries)


# ---- from the definitions, in 64 bits ------------------------------------------------------------


def _exact_keys(case, code, params):
    """Reconstructed keys of n pages of one head as complex numbers [n, 128, 64], x + i y."""
    low, wide = case["r_bits"], case["r_bits"] + case["t_bits"]
    bits = ((code[..., None].int() >> torch.arange(8, device=DEVICE)) & 1).flatten(-2)              # [n, 4, 128, bits of a unit]
    symbol = (bits.view(-1, BLOCKS, GROUP, 16, wide) << torch.arange(wide, device=DEVICE)).sum(-1).permute(0, 2, 1, 3).reshape(-1, GROUP, PAIRS)
    p = params.double().view(code.shape[0], -1, 1, PAIRS, 2)
    turn = (symbol >> low).double() + 0.5
    turn = turn * p[:, 1, ..., 0] + p[:, 1, ..., 1] if case["grouped_angles"] else turn * (math.tau / 2 ** case["t_bits"]) - math.pi
    return torch.polar((symbol % 2 ** low + 0.5).double() * p[:, 0, ..., 0] + p[:, 0, ..., 1], turn)


def _exact_values(case, values, params):
    """Values [n, 128, 128] of n pages of one head."""
    if case["v_bits"] == 16:
        return values.double()
    b = case["v_bits"]
    found = torch.zeros((values.shape[0], GROUP, HEAD_DIM), dtype=torch.float64, device=DEVICE)
    words = values.view(torch.int32).view(values.shape[0], -1, 16, 4)                               # [page, block, slice, word]
    per = 16 // b
    for token in range(per):
        for dim in range(8):
            word = 2 * (token // 2) + dim // 4 if b == 4 else token // 2
            shift = 16 * (token % 2) + b * (dim % 4 if b == 4 else dim)
            found[:, token::per, dim::8] = ((words[..., word] >> shift) & (2 ** b - 1)).double()
    return found * params[..., :1].double() + params[..., 1:].double()


def _exact_attention(case, state, seq, head, queries, chosen, length):
    """One KV head's outputs [group, d] and page weights [n] over `chosen` pages of the pools, the last of which ends with the sequence."""
    keys = _exact_keys(case, state["codes"][chosen, head], state["params"][chosen, head])
    values = _exact_values(case, state["v_pool"][chosen, head], None if state["v_params"] is None else state["v_params"][chosen, head])
    rest = length % GROUP
    if state["residual"] is not None and rest:
        tail = state["residual"][seq, head].double()
        keys[-1] = torch.complex(tail[:, :PAIRS], tail[:, PAIRS:])
    tokens = len(chosen) * GROUP - (GROUP - rest if rest else 0)
    k, v = keys.flatten(0, 1)[:tokens], values.flatten(0, 1)[:tokens]
    q = queries.double()
    logits = (torch.complex(q[:, :PAIRS], q[:, PAIRS:]).conj() @ k.t().contiguous()).real / math.sqrt(HEAD_DIM)
    weight = torch.softmax(logits, dim=-1)
    pages = torch.zeros(len(chosen) * GROUP, dtype=torch.float64, device=DEVICE)
    pages[:tokens] = weight.sum(0)
    return weight @ v, pages.view(-1, GROUP).sum(-1)


def exact(case, seed):
    """Scales, attention outputs and weights in float64; what is chosen is whole numbers that have no other value."""
    op = case["op"]
    if op == "select":
        return None
    state = prepare(case, seed)
    before, after = _lengths(case)
    if op == "evict":
        kept = torch.zeros(state["weights"].shape, dtype=torch.float64)
        for s, (row, n) in enumerate(zip(state["weights"].tolist(), after)):
            pages, ends = _pages_up(n), max(case["last"], 1 if n % GROUP else 0)
            gone = max(0, pages - max(case["kept"], min(pages, case["first"] + ends)))
            out = set(sorted(range(case["first"], pages - ends), key=lambda p: (row[p], p))[:gone])
            left = [row[p] for p in range(pages) if p not in out]
            kept[s, :len(left)] = torch.tensor(left, dtype=torch.float64)
        return [None, None, kept.to(DEVICE), None, None]
    heads, group = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    table = state["block_table"].tolist()
    if op == "bound":
        scales = state["bound_scales"].double()
        for s, (b, a) in enumerate(zip(before, after)):
            done = table[s][b // GROUP:a // GROUP]
            for h in range(heads if done else 0):
                k = _exact_keys(case, state["codes"][done, h], state["params"][done, h])
                scales[done, h] = torch.maximum(k.real.abs(), k.imag.abs()).amax(1).view(-1, BLOCKS, 16).amax(-1) / 127.0
        return [None, scales]
    out = torch.zeros((case["seqs"], case["q_heads"], HEAD_DIM), dtype=torch.float64, device=DEVICE)
    if op == "weights":
        weights = state["weights"].double()
        for s, n in enumerate(after):
            total = torch.zeros(_pages_up(n), dtype=torch.float64, device=DEVICE)
            for h in range(heads):
                mine = slice(h * group, (h + 1) * group)
                out[s, mine], of_head = _exact_attention(case, state, s, h, state["q"][s, mine], table[s][:_pages_up(n)], n)
                total += of_head
            weights[s, :_pages_up(n)] = total + case["decay"] * state["weights_before"][s, :_pages_up(n)].double()
        return [out, weights]
    # the choice is one of 32-bit numbers, whose products and sums are rounded one by one
    bounds, scales, q = state["bounds"].cpu().numpy(), state["bound_scales"].cpu().numpy(), state["q"].float().cpu().numpy()
    for s, n in enumerate(after):
        pages = _pages_up(n)
        held = table[s][:pages]
        for h in range(heads):
            mine = slice(h * group, (h + 1) * group)
            chosen = list(range(pages))
            if pages > case["chosen"]:
                best = _exact_scores(bounds[held, h], scales[held, h], q[s, mine])
                others = sorted(range(case["first"], pages - case["last"]), key=lambda p: (-best[p], p))
                others = others[:case["chosen"] - case["first"] - case["last"]]
                chosen = sorted([*range(case["first"]), *others, *range(pages - case["last"], pages)])
            out[s, mine] = _exact_attention(case, state, s, h, state["q"][s, mine], [held[p] for p in chosen], n)[0]
    return [out, None, None]


def _exact_scores(bounds, scales, q):
    """A head's page scores: bounds [pages, 4, 2, 32] and scales [pages, 4] of its pages, q [group, 128] of its queries."""
    pages = bounds.shape[0]
    terms = []
    for b in range(BLOCKS):
        part = q[:, [*range(16 * b, 16 * b + 16), *range(PAIRS + 16 * b, PAIRS + 16 * b + 16)]]
        largest = abs(part).max()
        code = (part * (part.dtype.type(127) / largest)).round() if largest >= TINY else part * 0
        number = code.astype("int64") @ bounds[:, b, 0].T.astype("int64") + abs(code).astype("int64") @ bounds[:, b, 1].T.astype("int64")
        terms.append(number.astype("float32") * (largest * scales[:, b]).reshape(1, pages))
    return ((terms[0] + terms[1]) + (terms[2] + terms[3])).max(axis=0).tolist()
