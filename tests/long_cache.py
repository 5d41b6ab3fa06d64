"""What the calls for long caches under a budget of pages should give, in NumPy: bounds, scores and choices in fp32, one rounding an
operation, as their definitions say; evictions; page weights in float64 of what a cache of chunks.py holds."""
import numpy as np
import torch

from chunks import G
from oracle import cache_format

F32 = np.float32


def bounds_of(codes, params, bits):
    """codes [n, H, 4, 128, unit] and params of complete pages -> int8 [n, H, 4, 64], fp32 [n, H, 4]."""
    n, heads = codes.shape[:2]
    r, t = bits
    found = cache_format.unpack_pages(codes, params, n * G, r, t)
    a, c = (x.reshape(n, G, heads, 64) for x in found[:2])
    s, z = (x.astype(F32)[:, None] for x in found[2:4])
    rho = (c.astype(F32) + F32(0.5)) * s + z                             # the product is exact
    theta = a + 0.5
    if len(found) > 4:
        theta = theta * found[4].astype(np.float64)[:, None] + found[5].astype(np.float64)[:, None]
    else:
        theta = theta * (2 * np.pi / 2 ** t) - np.pi
    x, y = rho * np.cos(theta).astype(F32), rho * np.sin(theta).astype(F32)
    e = np.stack([x, y], axis=-1).reshape(n, G, heads, 4, 16, 2).transpose(0, 2, 3, 5, 4, 1)     # [n, H, block, xy, 16, token]
    low, high = e.min(-1), e.max(-1)
    largest = np.maximum(abs(low), abs(high)).max((-1, -2))              # [n, H, block]
    with np.errstate(divide="ignore", over="ignore"):
        up = np.where(largest >= F32(2.0 ** -100), F32(127) / largest, F32(0)).astype(F32)[..., None, None]
    c8 = np.rint((low + high) * F32(0.5) * up).astype(np.int8)
    w8 = np.rint((high - low) * F32(0.5) * up).astype(np.int8)
    return np.concatenate([c8.reshape(n, heads, 4, 32), w8.reshape(n, heads, 4, 32)], -1), (largest / F32(127)).astype(F32)


def scores_of(q, bounds, scales):
    """q fp32 [group, 128] of one KV head, bounds [P, 4, 64], scales [P, 4] of its pages -> fp32 [P]."""
    terms = []
    for b in range(4):
        part = np.concatenate([q[:, 16 * b:16 * b + 16], q[:, 64 + 16 * b:80 + 16 * b]], -1).astype(F32)
        m = abs(part).max()
        up = F32(127) / m if m >= F32(2.0 ** -100) else F32(0)
        q8 = np.rint(part * up).astype(np.int64)
        n = q8 @ bounds[:, b, :32].T.astype(np.int64) + abs(q8) @ bounds[:, b, 32:].T.astype(np.int64)
        terms.append(n.astype(F32) * (m * scales[:, b])[None])
    return ((terms[0] + terms[1]) + (terms[2] + terms[3])).max(0)


def choice(scores, pages, n_selected, n_first, n_last):
    """Chosen page numbers in order."""
    if pages <= n_selected:
        return list(range(pages))
    others = range(n_first, pages - n_last)
    best = sorted(others, key=lambda p: (-scores[p], p))[:n_selected - n_first - n_last]
    return sorted([*range(n_first), *best, *range(pages - n_last, pages)])


def select(q, bounds, scales, table, lens, heads, n_selected, n_first, n_last):
    """selected [S, H, n_selected] and selected_lens [S, H]."""
    group = q.shape[1] // heads
    out, out_lens = np.full((len(lens), heads, n_selected), -1, np.int32), np.zeros((len(lens), heads), np.int32)
    n_pool = bounds.shape[0]
    for s, length in enumerate(lens):
        length = max(0, length)
        pages = (length + G - 1) // G
        ids = table[s, :pages]
        there = (ids >= 0) & (ids < n_pool)
        for h in range(heads):
            scores = np.zeros(pages, F32)
            if pages > n_selected:
                scores = np.where(there, scores_of(q[s, h * group:(h + 1) * group], bounds[np.where(there, ids, 0), h], scales[np.where(there, ids, 0), h]), -np.inf)
            chosen = choice(scores, pages, n_selected, n_first, n_last)
            out[s, h, :len(chosen)] = [ids[p] * heads + h if there[p] else -1 for p in chosen]
            out_lens[s, h] = length - (pages - len(chosen)) * G
    return out, out_lens


def evict(table, lens, weights, n_kept, n_first, n_last):
    """table, lens, weights afterwards, and the freed entries."""
    table, weights, lens, freed = table.copy(), weights.copy(), list(lens), []
    for s, length in enumerate(lens):
        length = max(0, length)
        pages = (length + G - 1) // G
        lens[s] = length
        if pages > table.shape[1]:
            continue
        last = max(n_last, 1 if length % G else 0)
        gone = max(0, pages - max(n_kept, min(pages, n_first + last)))
        w = np.where(np.isnan(weights[s]), np.inf, weights[s])
        nan = np.isnan(weights[s])
        order = sorted(range(n_first, pages - last), key=lambda p: (nan[p], w[p], p))[:gone]
        kept = [p for p in range(pages) if p not in set(order)]
        freed += [table[s, p] for p in sorted(order)]
        for row, nothing in ((table, -1), (weights, 0.0)):
            row[s, :pages] = list(row[s, kept]) + [nothing] * gone
        lens[s] = length - gone * G
    return table, np.array(lens, np.int32), weights, np.array(freed, np.int32)


def page_weights(cache, s, q):
    """float64 sums of the softmax weights by page over all heads of sequence s of a Cache, q [heads, d]; and each head's largest sum over the pairs
    of |q_j| |k~_j| times the scale, which bounds what relative errors of factors move a score by."""
    k = cache.k64[s]
    group = q.shape[0] // cache.heads
    pages = (k.shape[0] + G - 1) // G
    total, most = torch.zeros(pages * G, dtype=torch.float64, device=k.device), 0.0
    for h in range(q.shape[0]):
        kh, qh = k[:, h // group], q[h].double()
        w = torch.softmax((kh * qh).sum(-1) * cache.sm_scale, 0)
        total[:len(w)] += w
        most = max(most, float(((kh * qh).abs().sum(-1)).max()) * abs(float(cache.sm_scale)))
    return total.view(pages, G).sum(-1), most


def weight_tolerance(want, most, heads):
    """Bound of a page weight's error.  A weight is exp(score - top) / sum: factors of a score carry 22 bits each (two of them) and up to 64
    products are summed in fp32, so that a score is off by at most (2 * 2^-22 + 2^-20) * most (the sum of its terms' sizes), the score and the top each; it is
    rounded twice more in fp32, to 2^-23 of up to 2 * most; the exponential is good to 2^-22, and sums and quotient add 64 * 2^-24."""
    step = (2 * 2.0 ** -22 + 2.0 ** -20) * most * 2 + 2 * 2.0 ** -23 * 2 * most + 2.0 ** -22 + 64 * 2.0 ** -24
    return step * want + heads * 1e-12


def output_bar(spread, slope, want, most):
    """Bound of |error| / |output| of fp32 attention over values that enter exactly.  An output moves by the 2-norm over the tokens of weight times value
    (`spread`) for independent relative errors of the weights, which are the scores' absolute ones.  In the mean of squares: a pair's product has
    factors of 22 bits, two roundings of 2^-22 / sqrt(3) each at most, together below 2^-22 of it, and pairs add as squares (`slope`: their 2-norm, scaled); a sum of 64 pairs
    by parts is rounded at most 16 times where all of it is under way, by 2^-24 / sqrt(3) of at most the terms' sizes (`most`): below 2^-22 of that, too."""
    step = 2.0 ** -22 * (float(slope.max()) + most) + 2.0 ** -22
    return step * float(spread.norm()) / float(want.norm()) + 2.0 ** -22
