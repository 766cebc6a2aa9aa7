"""What the microscaled operators' compiled Python calls hand to the C entry points: the entries are replaced by callbacks
that write down their arguments, the tensors by stand-ins, so no device is needed."""
import ctypes as C

import pytest
import torch

TYPES = (torch.float32, torch.bfloat16, torch.float16)
P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
ARGUMENTS = (
    (P, I32, I64, I64, I64, I32, P, P, P, I64, P),                                           # quantize
    (I32, P, P, I64, I64, P, I32, I64, P),                                                   # dequantize
    (P, P, I32, I64, I64, I64, I64, P, I32, C.c_float, I32, P, P, P, I64, P, I64, P),        # rmsnorm_quantize
    (I32, P, P, I64, P, P, I64, I64, P, I32, I64, P),                                        # matmul
    (P, I32, I64, I64, I64, I32, P, P, I64, P, I32, I64, P, P),                              # linear
)


class Stand:
    """A tensor as far as the calls look at one: a CUDA tensor by its own account, its address never followed."""

    def __init__(self, shape, stride=None, dtype=torch.bfloat16, address=1 << 12):
        self.shape, self.dtype, self.address = torch.Size(shape), dtype, address
        self.strides = tuple(torch.empty(shape, device="meta").stride() if stride is None else stride)
        self.nbytes = self.shape.numel() * dtype.itemsize

    def stride(self):
        return self.strides

    def get_device(self):
        return 0

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return torch.empty_strided(self.shape, self.strides, device="meta").is_contiguous()


def held(rows, k, bits=4):
    """(codes, scales) of a [rows, k] matrix."""
    return (Stand((rows, -(-k // 128) * 16 * bits), dtype=torch.uint8),
            Stand((-(-rows // 128) * -(-k // 128) * 512,), dtype=torch.uint8))


@pytest.fixture()
def calls():
    """(the compiled calls, the list that their entries write to)"""
    from paper_2511_04063_b200 import build
    build.build()
    from paper_2511_04063_b200 import _calls
    seen = []

    def note(*args):
        seen.append(args)
        return 0

    entries = [C.CFUNCTYPE(I32, *a)(note) for a in ARGUMENTS]
    _calls.bind(tuple(C.cast(e, P).value for e in entries), TYPES, lambda: 0, lambda index: 0)
    yield _calls, seen         # (and the entries live until the test has ended)


@pytest.mark.parametrize("stride,ld", [((1, 1), 1), ((2, 2), 2), ((28, 7), 28), ((5000, 1), 5000), ((5000, 7), 5000)])
def test_one_column_keeps_its_row_stride(calls, stride, ld):
    """Every other column of a two-column matrix, a column of a three-dimensional one: the column's own stride says
    nothing, the rows' says where they are."""
    module, seen = calls
    x, other = Stand((100, 1), stride), Stand((100, 1), stride, address=1 << 16)
    module.quantize(x, 0, *held(100, 1), other, None)
    assert seen[-1][4] == ld and seen[-1][9] == ld
    module.dequantize(*held(100, 1), 0, x, None)
    assert seen[-1][7] == ld
    module.rmsnorm_quantize(x, None, 1e-5, 0, *held(100, 1), other, other, other, None)
    assert [seen[-1][i] for i in (5, 6, 14, 16)] == [ld] * 4
    module.matmul(*held(100, 64), 0, *held(1, 64), 64, x, None)
    assert seen[-1][10] == ld
    module.linear(x, 0, *held(1, 1), other, Stand((100 * 64 + 512,), dtype=torch.uint8), None)
    assert seen[-1][4] == ld and seen[-1][11] == ld


def test_strides_that_no_row_needs(calls):
    """One row may have any row stride; several rows neither overlap nor have gaps between their values."""
    module, seen = calls
    module.quantize(Stand((1, 64), (0, 1)), 0, *held(1, 64), None, None)
    assert seen[-1][4] == 64
    module.quantize(Stand((1, 1), (0, 7)), 0, *held(1, 1), None, None)
    assert seen[-1][4] == 1
    module.quantize(Stand((4, 64), (80, 1)), 0, *held(4, 64), None, None)
    assert seen[-1][4] == 80
    for shape, stride in (((4, 64), (0, 1)), ((4, 64), (63, 1)), ((4, 64), (128, 2)), ((1, 64), (128, 2)), ((4, 1), (0, 1)),
                          ((4, 1), (0, 7))):
        with pytest.raises(ValueError, match="contiguous"):
            module.quantize(Stand(shape, stride), 0, *held(*shape), None, None)


def test_the_self_tests_limits(calls):
    import paper_2511_04063_b200 as dq
    st, p = dq.load_library().dq_mx_selftest_bounded_wait, 1 << 12
    for step, limit in ((-1, 1000), (0, 0), (0, 10 ** 9)):
        assert st(0, p, p, 4, p, p, 64, 64, p, 1, 64, step, limit, None) == dq.DQ_ERR_INVALID_ARG
    assert st(0, p, p, 4, p, p, 64, 64, p, 1, 63, 0, 1000, None) == dq.DQ_ERR_INVALID_ARG
    assert st(0, p, p, 0, p, p, 64, 64, p, 1, 64, 0, 1000, None) == dq.DQ_OK


def test_rows_of_codes_are_counted_in_bytes(calls):
    """Two-dimensional codes have rows of their own; what counts is their bytes, whatever the elements' type."""
    module, seen = calls
    x, (codes, scales) = Stand((4, 256)), held(4, 256)               # rows of 128 bytes
    module.quantize(x, 0, Stand((4, 32), dtype=torch.int32), scales, None, None)
    module.quantize(x, 0, Stand((6, 128), dtype=torch.uint8), scales, None, None)
    module.quantize(x, 0, Stand((512,), dtype=torch.uint8), scales, None, None)
    module.quantize(x, 0, Stand((2, 2, 128), dtype=torch.uint8), scales, None, None)
    assert len(seen) == 4
    for shape, dtype in (((4, 128), torch.int16), ((4, 128), torch.float32), ((8, 64), torch.uint8), ((4, 256), torch.uint8),
                         ((2, 64), torch.int32)):
        with pytest.raises(ValueError, match="rows of 128 bytes"):
            module.quantize(x, 0, Stand(shape, dtype=dtype), scales, None, None)
    with pytest.raises(ValueError, match="at least"):
        module.quantize(x, 0, Stand((3, 128), dtype=torch.uint8), scales, None, None)
