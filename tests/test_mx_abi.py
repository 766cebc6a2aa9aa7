"""Host-side checks of the microscaled operators' entry points: sizes and refusals, which need no device."""
import pytest

import paper_2511_04063_b200 as dq


@pytest.fixture(scope="module")
def lib():
    from paper_2511_04063_b200 import build
    build.build()
    return dq.load_library()


def test_sizes(lib):
    assert dq.dq_mx_row_bytes(dq.DQ_MXFP4, 1) == 64 and dq.dq_mx_row_bytes(dq.DQ_MXFP4, 128) == 64
    assert dq.dq_mx_row_bytes(dq.DQ_MXFP8, 129) == 256
    assert dq.dq_mx_scale_bytes(1, 1) == 512 and dq.dq_mx_scale_bytes(129, 4096) == 2 * 32 * 512
    assert dq.dq_mx_linear_workspace(dq.DQ_MXFP4, 3, 200) == 3 * 128 + 2 * 512
    for bad in (dq.dq_mx_row_bytes(2, 128), dq.dq_mx_row_bytes(0, 0), dq.dq_mx_scale_bytes(-1, 8),
                dq.dq_mx_linear_workspace(0, 4, 1 << 25)):
        assert bad == -1


def test_refusals_come_before_any_cuda_call(lib):
    p, bad, big = 1 << 12, dq.DQ_ERR_INVALID_ARG, dq.DQ_ERR_UNSUPPORTED      # p: an aligned address that is never followed
    q = lib.dq_mx_quantize
    assert q(None, 0, 4, 64, 64, 0, p, p, None, 0, None) == bad
    assert q(p, 3, 4, 64, 64, 0, p, p, None, 0, None) == bad
    assert q(p, 0, 4, 64, 64, 2, p, p, None, 0, None) == bad
    assert q(p, 0, 4, 64, 63, 0, p, p, None, 0, None) == bad
    assert q(p, 0, -1, 64, 64, 0, p, p, None, 0, None) == bad
    assert q(p, 0, 4, 0, 64, 0, p, p, None, 0, None) == bad
    assert q(p, 0, 4, 64, 64, 0, None, p, None, 0, None) == bad
    assert q(p, 0, 4, 64, 64, 0, p, p, p, 63, None) == bad
    assert q(p + 1, 0, 4, 64, 64, 0, p, p, None, 0, None) == bad
    assert q(p, 0, 4, 64, 64, 0, p + 16, p, None, 0, None) == big
    assert q(p, 0, 4, 64, 64, 0, p, p + 8, None, 0, None) == big
    assert q(p, 0, 1 << 31, 64, 64, 0, p, p, None, 0, None) == big
    assert q(p, 0, 0, 64, 64, 0, None, None, None, 0, None) == dq.DQ_OK
    n = lib.dq_rmsnorm_quantize
    assert n(p, None, 1, 4, 64, 64, 0, p, 2, 1e-5, 1, p, p, None, 0, None, 0, None) == bad      # gamma: fp32 or X's type
    assert n(p, None, 1, 4, 64, 64, 0, None, 0, float("nan"), 1, p, p, None, 0, None, 0, None) == bad
    assert n(p, p, 1, 4, 64, 64, 63, None, 0, 1e-5, 1, p, p, None, 0, None, 0, None) == bad
    m = lib.dq_mx_matmul
    assert m(0, p, p, 4, p, p, 0, 64, p, 1, 64, None) == bad
    assert m(0, p, p, 4, p, p, 64, 64, p, 1, 63, None) == bad
    assert m(0, p, p, 4, p, p, 64, 64, None, 1, 64, None) == bad
    assert m(0, p, p, 4, p + 16, p, 64, 64, p, 1, 64, None) == big
    assert m(0, None, None, 0, p, p, 64, 64, None, 1, 64, None) == dq.DQ_OK
    li = lib.dq_mx_linear
    assert li(p, 1, 4, 64, 64, 0, p, p, 64, p, 1, 64, None, None) == bad
    assert li(p, 1, 4, 64, 64, 0, p, p, 64, p, 1, 64, p + 16, None) == big
    assert li(p, 1, 4, 64, 60, 0, p, p, 64, p, 1, 64, p, None) == bad


def test_compiled_calls_check_their_arguments(lib):
    """The Python calls' checks, with the lookups of device and stream replaced: no CUDA tensor, nothing is launched."""
    import ctypes as C

    import torch

    from paper_2511_04063_b200 import _calls
    names = ("dq_mx_quantize", "dq_mx_dequantize", "dq_rmsnorm_quantize", "dq_mx_matmul", "dq_mx_linear")
    entries = tuple(C.cast(getattr(lib, n), C.c_void_p).value for n in names)
    types = (torch.float32, torch.bfloat16, torch.float16)
    with pytest.raises(TypeError):
        _calls.bind(entries[:4], types, lambda: 0, lambda index: 0)
    _calls.bind(entries, types, lambda: 0, lambda index: 0)
    x, held = torch.zeros(4, 64), torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        _calls.quantize(x, 0, held, held, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        _calls.matmul(held, held, 0, held, held, 64, x, None)
    with pytest.raises(TypeError):
        _calls.linear(x)
    with pytest.raises(AttributeError):
        _calls.rmsnorm_quantize(None, None, 1e-5, 0, held, held, None, None, None, None)
