"""pq_chunk_attention loses no more than the roundings it is documented with.

A rounding to fp16 is off by 2^-11 of the value at most, and by U = 2^-11 / sqrt(3) in the mean of squares where the value is just above a power
of two (less elsewhere).  To first order a row's output is off by
    sum_t w_t (v_t - out) (ds_t + dp_t)  +  sum_t w_t v_t dv_t  +  out do,      ds_t = scale sum_j q_j k_tj dk_tj,
one dp for a weight (it is in the sum of weights as well: v - out), one dk for a key coordinate, two with the grouped quantizer (its levels are fp16, too),
one dv for a quantized value, none for an fp16 one, one do for the output.  They are independent, and values are on either side of zero, so that squares
add up:
    U^2 (sum_t w_t^2 (v_t - out)^2 (c scale^2 sum_j q_j^2 k_tj^2 + 1) + [values quantized] sum_t w_t^2 v_t^2 + out^2).
The sum over the rows and dims of a call holds some hundred independent contributions at least and stays below that: numbers spread evenly over a binade's
logarithm have 0.54 of it.  One bit less in the keys would be four times their part."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import DEV, Cache      # noqa: E402
from test_gpu_chunk_attention import _attend, _queries      # noqa: E402

U = 2.0 ** -11 / 3.0 ** 0.5


def _expected(c, s, q, positions, grouped, window, sinks):
    """(out, mean square of its error) in float64."""
    n, n_heads = q.shape[:2]
    k, v = c.k64[s], c.v64[s]
    token, position = torch.arange(k.shape[0], device=DEV), positions[:, None]
    seen = token <= position
    if window:
        seen &= (token > position - window) | (token < sinks)
    out, square = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for h in range(n_heads):
        kh, vh, qh = (x.contiguous() for x in (k[:, h * c.heads // n_heads], v[:, h * c.heads // n_heads], q[:, h].double()))
        w = torch.softmax((qh @ kh.t().contiguous() * c.sm_scale).masked_fill(~seen, -np.inf), dim=-1)
        out[:, h] = o = w @ vh
        slope = (2.0 if grouped else 1.0) * c.sm_scale ** 2 * ((qh * qh) @ (kh * kh).t().contiguous())
        a = w * w * (slope + 1.0)
        square[:, h] = a @ (vh * vh) - 2 * o * (a @ vh) + o * o * a.sum(-1, keepdim=True) + o * o
        if c.v_bits != 16:
            square[:, h] += (w * w) @ (vh * vh)
    return out, square * U * U


@pytest.mark.parametrize("bits,grouped", [((4, 4), False), ((3, 3), False), ((3, 5), False), ((4, 4), True), ((2, 4), True)])
@pytest.mark.parametrize("v_bits", [16, 4, 2])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("new,window,sinks", [([7, 5], 0, 0), ([160, 90], 0, 0), ([8, 6], 300, 4), ([150, 70], 300, 4)])
def test_errors_are_those_of_the_documented_roundings(bits, grouped, v_bits, tail, new, window, sinks):
    c = Cache([1500, 700], 2, bits, grouped, v_bits, tail, seed=11)
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _queries(int(starts[-1]), 8, 12)
    got = _attend(c, q, starts, window, sinks).double()
    error = expected = 0.0
    for s, n in enumerate(new):
        rows = slice(int(starts[s]), int(starts[s + 1]))
        out, square = _expected(c, s, q[rows], torch.arange(c.lens[s] - n, c.lens[s], device=DEV), grouped, window, sinks)
        error += float(((got[rows] - out) ** 2).sum())
        expected += float(square.sum())
    print(f"{bits} {grouped} v{v_bits} tail {tail} new {new} window {window}: {error / expected:.2f}", flush=True)
    assert error <= expected


def test_keys_of_a_tail_are_rounded_once():
    """A sequence of un-quantized keys only."""
    c = Cache([127, 120], 8, seed=3)
    q = _queries(160, 32, 4)
    got = _attend(c, q, [0, 100, 160]).double()
    error = expected = 0.0
    for s, rows, n in ((0, slice(0, 100), 100), (1, slice(100, 160), 60)):
        out, square = _expected(c, s, q[rows], torch.arange(c.lens[s] - n, c.lens[s], device=DEV), False, 0, 0)
        error += float(((got[rows] - out) ** 2).sum())
        expected += float(square.sum())
    assert error <= expected, error / expected
