"""The parameters of quantized values have to cover the pool that they belong to.  Refused before anything is launched: no GPU needed
for the Python functions' own checks (tensors of the host that say they are on the card)."""
import os

import pytest

torch = pytest.importorskip("torch")

import paper_2502_00527_amd as pq      # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(pq.lib_path()), reason="libpolarquant.so is not built")

D, G, HEADS, PAGES = 128, 128, 2, 3
SHORT = [(PAGES - 1, HEADS, G, 2), (PAGES, HEADS - 1, G, 2), (PAGES, HEADS, G), (PAGES * HEADS * G * 2 - 1,), (0,)]


class OnCard(torch.Tensor):
    is_cuda = property(lambda self: True)


def _tensor(shape, dtype):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnCard)


class _Declines:
    def __getattr__(self, name):
        return lambda *a: None


class _Library:
    """The library; calls that would launch something are noted instead."""

    def __init__(self):
        self.library, self.made = pq.load_library(), []

    def __getattr__(self, name):
        if "bytes" in name or name == "pq_strerror":
            return getattr(self.library, name)
        return lambda *a: self.made.append(name) or 0


def _calls(v_bits, v_params):
    i32, f16, u8 = torch.int32, torch.float16, torch.uint8
    lay = pq.Layout(D, 4, 4, G, HEADS, 0)
    codes, params, table, lens = _tensor((PAGES, HEADS, 4, G, 16), u8), _tensor((PAGES, HEADS, 64, 2), f16), _tensor((2, 2), i32), _tensor((2,), i32)
    v_pool = _tensor((PAGES, HEADS, G * v_bits // 16, 16, 16), u8)
    q, rows, starts, slots = _tensor((2, 4, D), f16), _tensor((2, HEADS, D), f16), _tensor((3,), i32), _tensor((2,), torch.int64)
    residual, space, out = _tensor((2, HEADS, G, D), f16), _tensor((1 << 20,), u8), _tensor((2, 4, D), torch.float32)
    common = (lay, q, codes, params, v_pool, table, lens, 200)
    return {
        "pq_append_chunk": (lay, rows, rows, starts, lens, slots, residual, table, codes, params, v_pool, v_bits, v_params),
        "pq_chunk_attention": (lay, q, starts, codes, params, v_pool, table, lens, 200, 0.1, _tensor((2, 4, D), f16), space, residual, v_bits, v_params),
        "pq_window_attention": (*common, 100, 4, 0.1, out, space, residual, v_bits, v_params),
        "pq_decode_attention": (*common, 0.1, out, space, None, residual, v_bits, v_params),
        "pq_decode_attention_static": (*common, 0.1, out, None, residual, v_bits, v_params),
        "pq_decode_partials": (*common, 0.1, space, None, residual, v_bits, v_params),
        "pq_encode_values": (lay, v_bits, rows, _tensor((1,), i32), v_pool, v_params),
    }


NAMES = list(_calls(4, None))


@pytest.mark.parametrize("v_bits", [4, 2])
@pytest.mark.parametrize("name", NAMES)
def test_short_parameters_are_refused(name, v_bits, monkeypatch):
    library = _Library()
    monkeypatch.setattr(pq, "_calls", _Declines())
    monkeypatch.setattr(pq, "_stream", lambda: 0)
    monkeypatch.setattr(pq, "load_library", lambda: library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    getattr(pq, name)(*_calls(v_bits, _tensor((PAGES, HEADS, G, 2), torch.float16))[name])
    assert library.made == [name]
    for shape in SHORT:
        with pytest.raises(pq.PolarQuantError, match="params holds"):
            getattr(pq, name)(*_calls(v_bits, _tensor(shape, torch.float16))[name])
    assert library.made == [name]


@pytest.mark.gpu
@pytest.mark.parametrize("v_bits", [4, 2])
def test_short_parameters_are_declined_and_refused(v_bits):
    """Through the native part, too, which only takes tensors of the card.  All lengths are zero."""
    native = pq._marshaller()
    for shape in [(PAGES, HEADS, G, 2), *SHORT]:
        for name, args in _calls(v_bits, _tensor(shape, torch.float16)).items():
            args = [torch.zeros(a.shape, dtype=a.dtype, device="cuda:0") if isinstance(a, torch.Tensor) else a for a in args]
            call = getattr(native, name[3:], None)
            if call is not None:
                more = [0, 0] if name == "pq_chunk_attention" else []
                assert call(*args, *more) == (None if shape in SHORT else 0), (name, shape)
            if shape in SHORT:
                with pytest.raises(pq.PolarQuantError, match="params holds"):
                    getattr(pq, name)(*args)
    torch.cuda.synchronize()
