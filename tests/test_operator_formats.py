"""The binding takes codes as bytes or as the format that the call names, scales as bytes: tensors of the other format are refused on the host."""
import pytest
import torch

from paper_2505_20524_amd import fog

DTYPE = {fog.E4M3: torch.float8_e4m3fn, fog.E5M2: torch.float8_e5m2}
FORMATS = (fog.E4M3, fog.E5M2)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def calls(fmt, q_type, s_type=torch.uint8):
    """Calls of every kind whose codes of format `fmt` are of q_type and whose scales are of s_type."""
    x, q, s = torch.zeros((4, 256), dtype=torch.bfloat16), u8(4, 256).view(q_type), u8(2, 4).view(s_type)
    s_col, tile, C = u8(1, 256).view(s_type), u8(1, 2).view(s_type), torch.zeros((4, 4), dtype=torch.bfloat16)
    byte = u8(4, 256)
    yield "rows", lambda: fog.quantize_block(x, fmt, q_row=q, s_row=s)
    yield "columns", lambda: fog.quantize_block(x, fmt, q_col=q, s_col=s_col)
    yield "tiles", lambda: fog.quantize_tile(x, fmt, q, tile)
    yield "A", lambda: fog.fp8_gemm_block(fog.NT, 4, 4, 256, q, fmt, fog.VECTOR, s, byte, 1 - fmt, fog.TILE, u8(1, 2), C)
    yield "B", lambda: fog.fp8_gemm_block(fog.NT, 4, 4, 256, byte, 1 - fmt, fog.VECTOR, u8(2, 4), q, fmt, fog.TILE, tile, C)
    if s_type == torch.uint8:
        yield "embedding", lambda: fog.embed_quantize(torch.zeros(4, dtype=torch.int64), x, 1.0, fmt, torch.ones(1), torch.zeros_like(x), q=q)


@pytest.fixture
def last_check(monkeypatch):
    """What is right so far is stopped where the device is looked at: nothing is launched on these host tensors."""
    class Stopped(Exception):
        pass

    def stop(*_):
        raise Stopped
    monkeypatch.setattr(fog, "_here", stop)
    return Stopped


@pytest.mark.parametrize("fmt", FORMATS)
def test_codes_of_the_other_format_are_refused(last_check, fmt):
    for what, call in calls(fmt, DTYPE[1 - fmt]):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(what)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("s_type", [torch.float8_e4m3fn, torch.float8_e5m2, torch.bool])
def test_scales_are_bytes(last_check, fmt, s_type):
    for what, call in calls(fmt, torch.uint8, s_type):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(what)


@pytest.mark.parametrize("fmt", FORMATS)
def test_codes_as_bytes_or_of_the_format_are_taken(last_check, fmt):
    for q_type in (torch.uint8, torch.int8, DTYPE[fmt]):
        for s_type in (torch.uint8, torch.int8):
            for _, call in calls(fmt, q_type, s_type):
                with pytest.raises(last_check):
                    call()
