"""Host-side checks of the key/value cache's operators: sizes and refusals of the C entry points, and what the compiled Python
calls check and hand on.  No device is needed: addresses are never followed, tensors are stand-ins."""
import ctypes as C

import pytest
import torch

import paper_2511_04063_b200 as dq

P, I32, I64, F = C.c_void_p, C.c_int32, C.c_int64, C.c_float
A = 1 << 12                                                    # an aligned address


@pytest.fixture(scope="module")
def lib():
    from paper_2511_04063_b200 import build
    build.build()
    return dq.load_library()


def heads(count=4, dim=128, address=A, token=None, head=None):
    return dq.dq_heads_t(address, count * dim if token is None else token, dim if head is None else head, count)


def cache(**over):
    v = dict(pages=A, n_pages=4, table=A, lengths=A, n_seqs=2, width=3, heads=2, dim=128, page=16)
    v.update(over)
    return dq.dq_kv_cache_t(*v.values())


def test_sizes_and_structs(lib):
    assert dq.dq_kv_page_bytes(16, 64) == 16 * 72 and dq.dq_kv_page_bytes(4096, 256) == 4096 * 264
    assert dq.dq_kv_attention_workspace(128) > 0 and dq.dq_kv_evict_workspace(2, 3, 10) == 2 * 3 * 24 * 4
    for bad in (dq.dq_kv_page_bytes(8, 128), dq.dq_kv_page_bytes(48, 128), dq.dq_kv_page_bytes(8192, 128), dq.dq_kv_page_bytes(16, 96),
                dq.dq_kv_attention_workspace(32), dq.dq_kv_evict_workspace(1, 0, 4), dq.dq_kv_evict_workspace(1, 1, 0)):
        assert bad == -1
    most = 2 ** 31 - 1
    assert dq.dq_kv_evict_workspace(most, 2, 4) == -1 and dq.dq_kv_evict_workspace(2 ** 30, 1, most) == -1
    assert dq.dq_kv_evict_workspace(2 ** 20, 1, most) == 2 ** 20 * (4 + 2 * most) * 4
    assert C.sizeof(dq.dq_heads_t) == 32 and C.sizeof(dq.dq_kv_cache_t) == 56
    assert dq.dq_heads_t.heads.offset == 24 and dq.dq_kv_cache_t.n_seqs.offset == 32


BAD, NOT_HERE, OK = dq.DQ_ERR_INVALID_ARG, dq.DQ_ERR_UNSUPPORTED, dq.DQ_OK


def rope(lib, q=None, k=None, dtype=1, tokens=3, dim=128, positions=A, freq=A, rot=128, qg=None, kg=None, g_type=1, eps=1e-6, flags=1,
         qo=None, ko=None):
    return lib.dq_qk_norm_rope(q or heads(), k, dtype, tokens, dim, positions, freq, rot, qg, kg, g_type, eps, flags, qo or heads(), ko, None)


def test_norm_and_rotation_refuse(lib):
    assert rope(lib, dtype=3) == BAD and rope(lib, tokens=-1) == BAD and rope(lib, rot=144) == BAD and rope(lib, flags=8) == BAD
    assert rope(lib, k=heads(2)) == BAD and rope(lib, k=heads(2), ko=heads(3)) == BAD and rope(lib, qo=heads(5)) == BAD
    assert rope(lib, positions=None) == BAD and rope(lib, freq=None) == BAD and rope(lib, positions=A + 2) == BAD
    assert rope(lib, eps=-1.0) == BAD and rope(lib, eps=float("nan")) == BAD and rope(lib, qg=A, g_type=2) == BAD
    assert rope(lib, qg=A, flags=0) == BAD and rope(lib, qg=A + 1) == BAD and rope(lib, q=heads(address=A + 1)) == BAD
    assert rope(lib, q=heads(address=None)) == BAD and rope(lib, q=heads(count=0)) == BAD and rope(lib, q=heads(head=100)) == BAD
    assert rope(lib, dim=72, rot=0) == NOT_HERE and rope(lib, q=heads(dim=272), qo=heads(dim=272), dim=272, rot=0) == NOT_HERE
    assert rope(lib, rot=24) == NOT_HERE and rope(lib, dim=96, rot=96, flags=5) == NOT_HERE and rope(lib, tokens=1 << 31) == NOT_HERE
    assert rope(lib, tokens=0) == OK


def append(lib, k=None, v=None, dtype=1, tokens=4, c=None, starts=None, kv=None, vv=None, positions=None, slots=None, ld=48):
    return lib.dq_kv_append(k or heads(2), v or heads(2), dtype, tokens, c or cache(), starts, kv, vv, positions, slots, ld, None)


def test_append_and_reading_back_refuse(lib):
    for over in (dict(n_seqs=-1), dict(heads=0), dict(width=0), dict(pages=None), dict(table=None), dict(lengths=None), dict(table=A + 2)):
        assert append(lib, c=cache(**over)) == BAD
    for over in (dict(dim=96), dict(page=24), dict(page=8), dict(pages=A + 64), dict(width=1 << 30)):
        assert append(lib, c=cache(**over)) == NOT_HERE
    assert append(lib, tokens=5) == BAD                          # no two equal parts
    assert append(lib, dtype=4) == BAD and append(lib, tokens=-2) == BAD and append(lib, tokens=1 << 31) == NOT_HERE
    assert append(lib, k=heads(3)) == BAD and append(lib, kv=heads(3)) == BAD and append(lib, starts=A + 1) == BAD
    assert append(lib, slots=A, ld=47) == BAD and append(lib, slots=A + 1) == BAD
    assert append(lib, tokens=0) == OK and append(lib, c=cache(n_seqs=0, table=None, lengths=None)) == OK
    read = lambda tokens=4, k=None, dtype=1: lib.dq_kv_dequantize(cache(), None, tokens, k or heads(2), heads(2), dtype, None)  # noqa: E731
    assert read(k=heads(4)) == BAD and read(tokens=3) == BAD and read(dtype=-1) == BAD and read(tokens=0) == OK


def attend(lib, q=None, dtype=1, tokens=4, c=None, starts=None, scale=0.1, out=None, lse=A, work=A):
    return lib.dq_kv_attention(q or heads(4), dtype, tokens, c or cache(), starts, scale, out or heads(4), lse, work, None)


def test_attention_weights_and_eviction_refuse(lib):
    assert attend(lib, dtype=0) == NOT_HERE and attend(lib, dtype=3) == BAD and attend(lib, q=heads(5), out=heads(5)) == BAD
    assert attend(lib, out=heads(2)) == BAD and attend(lib, scale=float("inf")) == BAD and attend(lib, scale=float("nan")) == BAD
    assert attend(lib, work=None) == BAD and attend(lib, work=A + 8) == NOT_HERE and attend(lib, lse=A + 2) == BAD
    assert attend(lib, tokens=0, work=None) == OK
    w = lambda tokens=4, lse=A, out=A, ld=48: lib.dq_kv_attention_weights(heads(4), 1, tokens, lse, cache(), None, 0.1, None, out, ld, None)  # noqa: E731
    assert w(lse=None) == BAD and w(out=None) == BAD and w(ld=40) == BAD
    e = lambda keep=4, recent=2, ld=48, work=A, lengths=A: lib.dq_kv_evict(cache(), A, A, ld, keep, recent, A, A, lengths, work, None)  # noqa: E731
    assert e(keep=0) == BAD and e(recent=-1) == BAD and e(recent=5) == BAD and e(ld=47) == BAD and e(work=None) == BAD
    assert e(lengths=None) == BAD and e(lengths=A + 1) == BAD
    assert lib.dq_kv_evict(cache(n_seqs=2 ** 30, heads=1), A, A, 48, 2 ** 31 - 1, 2, A, A, A, A, None) == NOT_HERE
    assert lib.dq_kv_evict(cache(n_seqs=0, table=None, lengths=None), A, A, 48, 4, 2, A, A, A, A, None) == OK


# ------------------------------------------------------------------------------------------------ the Python calls
class Stand:
    """A tensor as far as the calls look at one: a CUDA tensor by its own account, its address never followed."""

    def __init__(self, shape, stride=None, dtype=torch.bfloat16, address=A, device=0):
        self.shape, self.dtype, self.address, self.device_index = torch.Size(shape), dtype, address, device
        self.strides = tuple(torch.empty(shape, device="meta").stride() if stride is None else stride)
        self.nbytes = self.shape.numel() * dtype.itemsize

    def stride(self):
        return self.strides

    def get_device(self):
        return self.device_index

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return torch.empty_strided(self.shape, self.strides, device="meta").is_contiguous()


class Handle:
    def __init__(self, **over):
        self.struct = cache(**over)
        self._call = (C.addressof(self.struct), 0)


H, K = C.POINTER(dq.dq_heads_t), C.POINTER(dq.dq_kv_cache_t)
ENTRIES = (
    (H, H, I32, I64, I32, P, P, I32, P, P, I32, F, I32, H, H, P), (H, H, I32, I64, K, P, H, H, P, P, I64, P), (K, P, I64, H, H, I32, P),
    (H, I32, I64, K, P, F, H, P, P, P), (H, I32, I64, P, K, P, F, P, P, I64, P), (K, P, P, I64, I32, I32, P, P, P, P, P),
)


@pytest.fixture()
def calls(lib):
    from paper_2511_04063_b200 import _calls
    seen = []

    def entry(types):
        def note(*args):
            seen.append([(a.contents.token_stride, a.contents.head_stride, a.contents.heads) if isinstance(a, H) and a else a for a in args])
            return 0
        return C.CFUNCTYPE(I32, *types)(note)

    entries = [entry(t) for t in ENTRIES]
    mx = tuple(C.cast(getattr(lib, n), P).value for n in ("dq_mx_quantize", "dq_mx_dequantize", "dq_rmsnorm_quantize", "dq_mx_matmul", "dq_mx_linear"))
    _calls.bind(mx, (torch.float32, torch.bfloat16, torch.float16), lambda: 0, lambda index: 0)
    sizes = tuple(C.cast(getattr(lib, n), P).value for n in ("dq_kv_attention_workspace", "dq_kv_evict_workspace"))
    _calls.bind_kv(tuple(C.cast(e, P).value for e in entries) + sizes, torch.int32)
    yield _calls, seen


def i32(*shape, **kw):
    return Stand(shape, dtype=torch.int32, **kw)


def f32(*shape, **kw):
    return Stand(shape, dtype=torch.float32, **kw)


def test_strides_are_handed_on(calls):
    m, seen = calls
    fused = Stand((5, 4, 128), (1280, 128, 1))
    first = Stand((5, 4, 128), (128, 640, 1))
    m.attention(fused, Handle(n_seqs=5), 0.1, first, Stand((1 << 26,), dtype=torch.uint8), None, None, None)
    assert seen[-1][0] == (1280, 128, 4) and seen[-1][6] == (128, 640, 4) and seen[-1][2] == 5
    one = Stand((1, 4, 128), (0, 128, 1))                      # one token: its stride means nothing
    m.attention(one, Handle(n_seqs=1), 0.1, one, Stand((1 << 26,), dtype=torch.uint8), None, None, None)
    assert seen[-1][0][1:] == (128, 4) and seen[-1][0][0] >= 128
    for bad in (Stand((5, 4, 128), (512, 128, 2)), Stand((5, 4, 128), (512, 64, 1)), Stand((5, 4, 128), (0, 128, 1))):
        with pytest.raises(ValueError, match="contiguous|overlap"):
            m.attention(bad, Handle(n_seqs=5), 0.1, first, Stand((1 << 26,), dtype=torch.uint8), None, None, None)


def test_calls_refuse_what_does_not_fit(calls):
    m, seen = calls
    q, h, work = Stand((4, 4, 128)), Handle(), Stand((1 << 26,), dtype=torch.uint8)

    def refuses(match, call, *args):
        with pytest.raises(ValueError, match=match):
            call(*args)

    at = lambda **o: (m.attention, *{**dict(q=q, c=h, s=0.1, out=q, w=work, st=None, lse=None, stream=None), **o}.values())  # noqa: E731
    m.attention(*at()[1:])
    assert len(seen) == 1
    refuses("head_dim", *at(q=Stand((4, 4, 64)), out=Stand((4, 4, 64))))
    refuses("device", *at(q=Stand((4, 4, 128), device=1), out=Stand((4, 4, 128), device=1)))
    refuses("CUDA tensor", *at(q=Stand((4, 512))))
    refuses("CUDA tensor", *at(q=Stand((4, 4, 128), dtype=torch.float64)))
    refuses("differ", *at(out=Stand((5, 4, 128))))
    refuses("differ", *at(out=Stand((4, 4, 128), dtype=torch.float16)))
    refuses("heads", *at(out=Stand((4, 2, 128))))
    refuses("workspace", *at(w=Stand((1000,), dtype=torch.uint8)))
    refuses("starts", *at(st=i32(2)))
    refuses("starts", *at(st=Stand((3,), dtype=torch.int64)))
    refuses("starts", *at(st=i32(3, device=1)))
    refuses("lse", *at(lse=f32(4, 3)))
    with pytest.raises(AttributeError):
        m.attention(q, None, 0.1, q, work, None, None, None)
    with pytest.raises(TypeError):
        m.attention(q)

    x = Stand((4, 2, 128))
    m.append(x, x, h, None, None, x, i32(4), i32(2, 2, 50), None)
    assert seen[-1][10] == 50 and seen[-1][6] is None or not seen[-1][6]
    refuses("V", m.append, x, Stand((4, 2, 64)), h, None, None, None, None, None, None)
    refuses("heads", m.append, q, x, h, None, None, None, None, None, None)
    refuses("positions", m.append, x, x, h, None, None, None, i32(5), None, None)
    refuses("slot_positions", m.append, x, x, h, None, None, None, None, i32(2, 2, 40), None)
    refuses("heads", m.kv_dequantize, h, x, q, None, None)

    m.attention_weights(q, f32(4, 4), h, 0.1, f32(2, 2, 48), None, None, None)
    refuses("lse", m.attention_weights, q, f32(4, 5), h, 0.1, f32(2, 2, 48), None, None, None)
    refuses("weights_out", m.attention_weights, q, f32(4, 4), h, 0.1, i32(2, 2, 48), None, None, None)
    refuses("weights", m.attention_weights, q, f32(4, 4), h, 0.1, f32(2, 2, 48), f32(2, 2, 49), None, None)

    ev = lambda **o: (m.evict, *{**dict(c=h, w=f32(2, 2, 48), p=i32(2, 2, 48), keep=4, recent=1, wo=f32(2, 2, 48), po=i32(2, 2, 48),  # noqa: E731
                                        n=i32(2), work=work, stream=None), **o}.values())
    m.evict(*ev()[1:])
    refuses("positions", *ev(p=f32(2, 2, 48)))
    refuses("weights_out", *ev(wo=f32(2, 2, 64)))
    refuses("lengths_out", *ev(n=i32(3)))
    refuses("keep", *ev(keep=0))
    refuses("recent", *ev(recent=-1))
    refuses("workspace", *ev(work=Stand((100,), dtype=torch.uint8)))


def test_norm_and_rotation_calls(calls):
    m, seen = calls
    q, k = Stand((3, 4, 128)), Stand((3, 2, 128))
    ok = dict(q=q, k=k, p=i32(3), f=f32(64), qo=q, ko=k, qg=Stand((128,)), kg=Stand((128,)), eps=1e-6, flags=1, stream=None)
    run = lambda **o: m.qk_norm_rope(*{**ok, **o}.values())  # noqa: E731
    run()
    assert seen[-1][7] == 128 and seen[-1][10] == dq.DQ_BF16
    run(qg=f32(128), kg=None, f=f32(16))
    assert seen[-1][7] == 32 and seen[-1][10] == dq.DQ_FP32
    run(p=None, f=None, k=None, ko=None)
    assert seen[-1][7] == 0 and not seen[-1][1] and not seen[-1][14]
    for over, match in ((dict(ko=None), "both"), (dict(qo=k), "heads"), (dict(p=i32(4)), "positions"), (dict(f=f32(65)), "frequencies"),
                        (dict(f=Stand((64,))), "inv_freq"), (dict(qg=f32(128)), "gamma"), (dict(qg=Stand((64,))), "gamma"),
                        (dict(flags=-1), "flags"), (dict(p=Stand((3,), dtype=torch.int64)), "positions")):
        with pytest.raises(ValueError, match=match):
            run(**over)


def test_the_handle_checks_its_tensors(lib):
    pages, table, lengths = torch.zeros(4, 2, 16 * 136, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="pages"):
        dq.dq_kv_cache(pages, table, lengths, 128)               # not on a device
    with pytest.raises(ValueError, match="pages of"):
        dq.dq_kv_pages(4, 2, 96, 16)
    with pytest.raises(AttributeError, match="fixed"):
        dq.dq_kv_cache.__setattr__(object.__new__(dq.dq_kv_cache), "lengths", lengths)
