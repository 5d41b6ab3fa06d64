"""A paged cache for tests of chunks of new tokens: filled by the library's encoders (whose bytes other tests pin to the
oracle), read back with the oracle's unpacking, and attention over it in float64."""
import numpy as np
import torch

from oracle import cache_format, polar, values as ovalues

D, G = 128, 128
DEV = "cuda:0"


def layout(bits, heads, grouped=False):
    import paper_2502_00527_amd as pq
    return pq.Layout(D, bits[0], bits[1], G, heads, int(grouped))


def pools(pages, bits, heads, grouped, v_bits, poison=True):
    """codes, params, values and their parameters of a pool, poisoned so that what must not be read shows."""
    nan = float("nan") if poison else 0.0
    shape = (pages, heads, 2, 64, 2) if grouped else (pages, heads, 64, 2)
    codes = torch.full((pages, heads, 4, G, 2 * sum(bits)), 0xA5 if poison else 0, dtype=torch.uint8, device=DEV)
    params = torch.full(shape, nan, dtype=torch.float16, device=DEV)
    if v_bits == 16:
        return codes, params, torch.full((pages, heads, G, D), nan, dtype=torch.float16, device=DEV), None
    return (codes, params, torch.full((pages, heads, G * v_bits // 16, 16, 16), 0xC3 if poison else 0, dtype=torch.uint8, device=DEV),
            torch.full((pages, heads, G, 2), nan, dtype=torch.float16, device=DEV))


class Cache:
    """lens: tokens per sequence, all of them in the cache.  tail: the keys of a sequence's incomplete group are fp16 rows of the
    residual buffer; otherwise its page is packed.  Pages come in a random order, `spare` of the pool belong to nobody."""

    def __init__(self, lens, heads, bits=(4, 4), grouped=False, v_bits=16, tail=True, seed=0, key_scale=1.0, spare=3):
        import paper_2502_00527_amd as pq

        rng = np.random.default_rng(seed)
        self.pq, self.bits, self.v_bits, self.lens, self.heads = pq, bits, v_bits, list(lens), heads
        self.layout = layout(bits, heads, grouped)
        counts = [(n + G - 1) // G for n in self.lens]
        width = max(1, max(counts, default=1))
        order = rng.permutation(sum(counts) + spare).astype(np.int32)
        self.codes, self.params, self.v_pool, self.v_params = pools(len(order), bits, heads, grouped, v_bits)
        self.residual = torch.full((len(self.lens), heads, G, D), float("nan"), dtype=torch.float16, device=DEV) if tail else None
        table = np.full((len(self.lens), width), -1, np.int32)
        self.k64, self.v64 = [], []
        at = 0
        for s, L in enumerate(self.lens):
            ids = order[at:at + counts[s]]
            at += counts[s]
            table[s, :counts[s]] = ids
            keys = (rng.standard_normal((L, heads, D)) * key_scale).astype(np.float32)
            keys[:, :, 5] *= 8.0
            keys = keys.astype(np.float16)
            values = rng.standard_normal((L, heads, D)).astype(np.float16)
            k_hat = keys.astype(np.float64)
            packed = L // G * G if tail else L
            dev_ids = torch.from_numpy(ids.copy()).to(DEV)
            if packed:
                n = (packed + G - 1) // G
                pq.pq_encode_keys(self.layout, torch.from_numpy(keys[:packed]).to(DEV), dev_ids[:n], self.codes, self.params)
                a, c, *par = cache_format.unpack_pages(self.codes[dev_ids[:n].long()].cpu().numpy(), self.params[dev_ids[:n].long()].cpu().numpy(), packed, *bits)
                k_hat[:packed] = polar.dequant_keys(a, c, par[0], par[1], bits[1], G, *par[2:])
            if packed < L:
                self.residual[s, :, :L - packed] = torch.from_numpy(keys[packed:]).to(DEV).permute(1, 0, 2)
            v_hat = values.astype(np.float64)
            if L and v_bits == 16:
                rows = torch.full((counts[s] * G, heads, D), float("nan"), dtype=torch.float16, device=DEV)
                rows[:L] = torch.from_numpy(values).to(DEV)
                self.v_pool[dev_ids.long()] = rows.view(-1, G, heads, D).permute(0, 2, 1, 3)
            elif L:
                pq.pq_encode_values(self.layout, v_bits, torch.from_numpy(values).to(DEV), dev_ids, self.v_pool, self.v_params)
                code = cache_format.unpack_value_pages(self.v_pool[dev_ids.long()].cpu().numpy(), L, v_bits)
                par = self.v_params[dev_ids.long()].cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, heads, 2)[:L]
                v_hat = ovalues.dequant_values(code, par[..., 0], par[..., 1])
                if L % G:                                            # parameters behind the last token are never to be used
                    self.v_params[dev_ids[-1].long(), :, L % G:] = float("nan")
            self.k64.append(torch.from_numpy(np.asarray(k_hat, np.float64)).to(DEV))
            self.v64.append(torch.from_numpy(np.asarray(v_hat, np.float64)).to(DEV))
        self.table = table
        self.block_table = torch.from_numpy(table).to(DEV)
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.max_seq_len = max(1, max(self.lens, default=1))
        self.sm_scale = 1.0 / np.sqrt(D)

    def rows(self, s, q, positions, window=0, sinks=0, sm_scale=None):
        """(out, spread) in float64 of query rows q [n, query heads, d] at the given positions of sequence s: the attention, and the
        2-norm over the tokens of weight times value, which is what independent relative errors of the weights move it by."""
        scale = self.sm_scale if sm_scale is None else sm_scale
        n, n_heads = q.shape[:2]
        group = n_heads // self.heads
        k, v = self.k64[s], self.v64[s]
        out = torch.zeros((n, n_heads, D), dtype=torch.float64, device=DEV)
        spread, slope = torch.zeros_like(out), torch.zeros((n, n_heads), dtype=torch.float64, device=DEV)
        if k.shape[0] == 0:
            return out, spread, slope
        token = torch.arange(k.shape[0], device=DEV)
        position = torch.as_tensor(positions, device=DEV)[:, None]
        seen = token <= position
        if window:
            seen &= (token > position - window) | (token < sinks)
        for h in range(n_heads):
            kh, vh = k[:, h // group].contiguous(), v[:, h // group].contiguous()
            qh = q[:, h].double()
            scores = (qh @ kh.t().contiguous() * scale).masked_fill(~seen, -np.inf)
            top = scores.amax(-1, keepdim=True).nan_to_num(neginf=0.0)
            w = torch.exp(scores - top)
            w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
            out[:, h] = w @ vh
            spread[:, h] = ((w * w) @ (vh * vh)).sqrt()
            # 2-norm over the pairs of |q_j| |k~_j|, the largest over the tokens a row sees
            pairs_q = qh[:, :64] ** 2 + qh[:, 64:] ** 2
            pairs_k = kh[:, :64] ** 2 + kh[:, 64:] ** 2
            slope[:, h] = (pairs_q @ pairs_k.t().contiguous()).masked_fill(~seen, 0.0).amax(-1).sqrt() * abs(scale)
        return out, spread, slope


def tolerance(out, spread, slope):
    """Bound of |error| of an fp16 output whose keys, weights and values enter as fp16.  A rounding is off by 2^-11 of its value at
    most, 2^-11 / sqrt(3) in the mean of squares.  A key coordinate has three (table, product, sum), which move a score by slope *
    2^-11 in that mean; the weight and the value have one each: in all (slope + 2 / sqrt(3)) 2^-11 of each token's contribution, independent from token to
    token.  Eight times that, and the output's own rounding."""
    step = 2.0 ** -11
    return 8 * (slope[..., None] + 1.2) * step * spread + step * out.abs() + 1e-7
