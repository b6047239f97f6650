"""CPU checks of the types that hold 8-bit codes: what the binding lets through to the
library, which reads every byte as e4m3."""
import pytest

from test_abi import ss  # noqa: F401  (fixture: the built library)

torch = pytest.importorskip("torch")


@pytest.fixture
def calls(ss, monkeypatch):  # noqa: F811
    """The names of the calls that reach the library, of tensors on no GPU."""
    made = []
    monkeypatch.setattr(ss, "_same_device", lambda *a: 0)
    monkeypatch.setattr(ss, "_run", lambda where, *a: made.append(where))
    return made


OTHERS = ["float8_e5m2", "float8_e4m3fnuz", "float8_e5m2fnuz", "float8_e8m0fnu", "bool", "quint8", "qint8"]


def empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("rows", [1, 128])
def test_codes_of_another_type_are_refused(ss, calls, rows):  # noqa: F811
    """A tensor of e5m2 or of a biased e4m3 would mean other values to its reader."""
    x, scales = empty((4, 256), torch.float16), empty((4 if rows == 1 else 1, 2), torch.float32)
    for name in OTHERS:
        if not hasattr(torch, name):
            continue
        codes = empty((4, 256), getattr(torch, name))
        for f in (lambda: ss.fp8_quantize(x, codes, scales, rows=rows), lambda: ss.fp8_dequantize(codes, scales, x, rows=rows),
                  lambda: ss.make_fp8(codes, empty((1, 2), torch.float32))):
            with pytest.raises(ss.SwiftSpecError) as e:
                f()
            assert e.value.status == ss.INVALID_ARG, name
    assert calls == []


@pytest.mark.parametrize("rows", [1, 128])
def test_bytes_and_e4m3_are_taken(ss, calls, rows):  # noqa: F811
    x, scales = empty((4, 256), torch.float16), empty((4 if rows == 1 else 1, 2), torch.float32)
    for dtype in (torch.uint8, torch.int8, torch.float8_e4m3fn):
        codes = empty((4, 256), dtype)
        ss.fp8_quantize(x, codes, scales, rows=rows)
        ss.fp8_dequantize(codes, scales, x, rows=rows)
        ss.make_fp8(codes, empty((1, 2), torch.float32))
    assert calls == ["fp8_quantize", "fp8_dequantize"] * 3
