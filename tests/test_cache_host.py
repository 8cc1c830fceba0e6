"""Host-side checks of the cache's calls (s2o_decode, s2o_key_weights, s2o_evict) that need no GPU: struct layouts, size queries and
refusals, all before any HIP call, and the binding's own checks of tensors."""
import ctypes as C

import pytest
import torch

from paper_2602_22575_amd import binding as b

FAKE = C.c_void_p(0x100000)
BIG = 1 << 60


@pytest.fixture(scope="module")
def lib():
    return b.load_library()


def test_struct_layouts():
    assert C.sizeof(b.S2ODecodeParams) == 12 * 4 + (4 + 3 + 3 + 4 + 4 + 4) * 8
    assert C.sizeof(b.S2OWeightsParams) == 12 * 4 + (4 + 3) * 8
    assert C.sizeof(b.S2OEvictParams) == 10 * 4 + 12 * 8


DECODE = dict(Z=1, B=2, H=4, Hkv=2, D=128, T=1, L=1000, own_len=10)
WEIGHTS = dict(Z=1, B=2, H=4, Hkv=2, D=128, T=3, L=1000)
EVICT = dict(Z=1, Hkv=2, D=128, L=1000, keep=100)
COMMON = [
    (dict(Z=0), b.S2O_EINVAL), (dict(Hkv=0), b.S2O_EINVAL), (dict(D=0), b.S2O_EINVAL), (dict(D=96), b.S2O_EUNSUPPORTED), (dict(D=256), b.S2O_EUNSUPPORTED),
    (dict(L=-1), b.S2O_EINVAL), (dict(L=(1 << 30) + 1), b.S2O_EUNSUPPORTED),
    (dict(k_stride=(1 << 20, 1 << 18, 100)), b.S2O_EINVAL),              # not a multiple of 8
    (dict(k_stride=(1 << 20, 1 << 18, 64)), b.S2O_EINVAL),               # a row stride shorter than a row
    (dict(k_stride=(1 << 20, -(1 << 18), 128)), b.S2O_EINVAL),
    (dict(k_stride=(1 << 62, 1 << 62, 128), Z=8, Hkv=4), b.S2O_EINVAL),  # beyond 64 bits
    (dict(k_stride=(1 << 40, 1 << 36, 1 << 23)), b.S2O_EUNSUPPORTED),    # a row stride of 16 MiB
]
QUERIES = [
    (dict(B=0), b.S2O_EINVAL), (dict(T=0), b.S2O_EINVAL), (dict(H=5), b.S2O_EINVAL),
    (dict(softmax_scale=-1.0), b.S2O_EINVAL), (dict(softmax_scale=float("nan")), b.S2O_EINVAL), (dict(softmax_scale=float("inf")), b.S2O_EINVAL),
    (dict(q_stride=(1 << 20, 1 << 18, 100, 8)), b.S2O_EINVAL),
    (dict(B=1 << 20, T=1 << 12), b.S2O_EUNSUPPORTED), (dict(Z=1 << 24), b.S2O_EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", COMMON + QUERIES + [
    (dict(L=0, own_len=0), b.S2O_EINVAL), (dict(own_len=-1), b.S2O_EINVAL), (dict(own_len=(1 << 30) + 1), b.S2O_EUNSUPPORTED),
    (dict(own_v_stride=(1 << 20, 1 << 18, 1 << 16, 100)), b.S2O_EINVAL),
    (dict(o_stride=(0, 512, 64, 128)), b.S2O_EINVAL),                    # rows of O overlap
    (dict(o_stride=(0, 0, 128, 128)), b.S2O_EINVAL),                     # two sequences write the same rows
])
def test_decode_refuses(kw, code):
    with pytest.raises(b.S2OError) as e:
        b.s2o_decode_sizes(b.make_decode_params(**{**DECODE, **kw}))
    assert e.value.code == code


@pytest.mark.parametrize("kw,code", COMMON + QUERIES + [(dict(L=0), b.S2O_EINVAL), (dict(causal=2), b.S2O_EINVAL)])
def test_weights_refuses(kw, code):
    with pytest.raises(b.S2OError) as e:
        b.s2o_key_weights_sizes(b.make_weights_params(**{**WEIGHTS, **kw}))
    assert e.value.code == code


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(L=0), b.S2O_EINVAL), (dict(keep=0), b.S2O_EINVAL), (dict(keep=1001), b.S2O_EINVAL), (dict(sink=-1), b.S2O_EINVAL),
    (dict(recent=-1), b.S2O_EINVAL), (dict(sink=60, recent=41), b.S2O_EINVAL),
    (dict(out_k_stride=(1 << 20, 64, 128)), b.S2O_EINVAL),               # rows of K_out overlap
    (dict(out_v_stride=(1 << 20, 0, 128)), b.S2O_EINVAL),
])
def test_evict_refuses(kw, code):
    with pytest.raises(b.S2OError) as e:
        b.s2o_evict_sizes(b.make_evict_params(**{**EVICT, **kw}))
    assert e.value.code == code


def test_wrong_struct_size_or_reserved_word(lib):
    for p, fn in ((b.make_decode_params(**DECODE), lambda p: lib.s2o_decode_sizes(C.byref(p), None, None)),
                  (b.make_weights_params(**WEIGHTS), lambda p: lib.s2o_key_weights_sizes(C.byref(p), 0, None, None)),
                  (b.make_evict_params(**EVICT), lambda p: lib.s2o_evict_sizes(C.byref(p), None))):
        assert fn(p) == b.S2O_OK
        p.reserved = 1
        assert fn(p) == b.S2O_EINVAL
        p.reserved, p.struct_size = 0, p.struct_size - 8
        assert fn(p) == b.S2O_EINVAL
    assert lib.s2o_decode_sizes(None, None, None) == b.S2O_EINVAL


def test_strides_of_single_dimensions_are_not_looked_at():
    b.s2o_decode_sizes(b.make_decode_params(1, 1, 4, 4, 128, 1, 1000, q_stride=(3, 7, 128, 5), o_stride=(0, 1, 128, 9), k_stride=(1, 128000, 128)))


def test_sizes():
    sz = b.s2o_decode_sizes(b.make_decode_params(1, 32, 32, 8, 128, 1, 32768, 512))
    assert sz["lse"] == 32 * 32 * 4 and sz["scratch"] >= 2 * 32 * 32 * (128 + 2) * 4
    assert b.s2o_decode_sizes(b.make_decode_params(1, 2, 8, 2, 128, 1, 96, 24))["scratch"] == 0
    w = b.make_weights_params(1, 1, 32, 8, 128, 64, 131072, causal=1)
    assert b.s2o_key_weights_sizes(w)["weights"] == 8 * 131072 * 4
    assert b.s2o_key_weights_sizes(w)["scratch"] >= 32 * 64 * 8                     # the rows' statistics
    assert b.s2o_key_weights_sizes(w, with_lse=True)["scratch"] <= b.s2o_key_weights_sizes(w)["scratch"]


def _refused(fn, args, cases):
    for i, bad, code in cases:
        a = list(args)
        a[i] = bad
        assert fn(*a) == code, (i, bad)


def test_decode_pointers(lib):
    p = b.make_decode_params(1, 2, 4, 2, 128, 1, 100000, 10)
    args = [FAKE] * 7 + [C.byref(p), FAKE, FAKE, FAKE, BIG, None]
    odd = C.c_void_p(0x100008)
    _refused(lib.s2o_decode, args, [(i, None, b.S2O_EINVAL) for i in (0, 1, 2, 3, 4, 7, 8)] + [(i, odd, b.S2O_EINVAL) for i in (0, 1, 2, 3, 4, 8)] +
             [(i, C.c_void_p(0x100002), b.S2O_EINVAL) for i in (5, 6, 9)] +
             [(10, None, b.S2O_ESCRATCH), (10, C.c_void_p(0x100080), b.S2O_ESCRATCH), (11, 256, b.S2O_ESCRATCH)])


def test_weights_pointers(lib):
    p = b.make_weights_params(1, 1, 4, 2, 128, 64, 100000, causal=1)
    args = [FAKE, FAKE, None, None, C.byref(p), None, FAKE, FAKE, BIG, None]
    two = C.c_void_p(0x100002)
    _refused(lib.s2o_key_weights, args, [(i, None, b.S2O_EINVAL) for i in (0, 1, 4, 6)] + [(i, two, b.S2O_EINVAL) for i in (0, 1, 2, 3, 5, 6)] +
             [(5, C.c_void_p(0x100004), b.S2O_EINVAL),                              # prev overlaps weights, shifted
              (7, None, b.S2O_ESCRATCH), (7, C.c_void_p(0x100080), b.S2O_ESCRATCH), (8, 16, b.S2O_ESCRATCH)])


def test_evict_pointers(lib):
    p = b.make_evict_params(1, 2, 128, 1000, 100)
    at = [C.c_void_p((i + 1) << 24) for i in range(9)]
    args = [at[0], at[1], at[2], at[3], C.byref(p), at[4], at[5], at[6], at[7], at[8], None, 0, None]
    refused = [(i, None, b.S2O_EINVAL) for i in (0, 1, 2, 4, 5, 6, 8)]               # (K without K_out and the other way round)
    refused += [(i, C.c_void_p(at[0].value + 8), b.S2O_EINVAL) for i in (0, 1, 5, 6)]
    refused += [(i, C.c_void_p((20 << 24) + 2), b.S2O_EINVAL) for i in (2, 3, 7, 8, 9)]
    refused += [(5, at[0], b.S2O_EINVAL), (5, C.c_void_p(at[0].value + 1024), b.S2O_EINVAL), (6, at[1], b.S2O_EINVAL),    # in place
                (6, at[4], b.S2O_EINVAL), (7, at[2], b.S2O_EINVAL), (8, at[6], b.S2O_EINVAL), (9, at[3], b.S2O_EINVAL), (8, at[2], b.S2O_EINVAL)]
    _refused(lib.s2o_evict, args, refused)


# ---- the binding's own checks come before the library is called (CPU tensors are refused like any other stray one)
def test_binding_refuses_cpu_tensors():
    q, k = torch.zeros(1, 2, 4, 1, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 1000, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="Q"):
        b.s2o_decode(q, k, k, b.make_decode_params(1, 2, 4, 2, 128, 1, 1000))
    with pytest.raises(ValueError, match="Q"):
        b.s2o_key_weights(q, k, b.make_weights_params(1, 2, 4, 2, 128, 1, 1000))
    w = torch.zeros(1, 2, 1000)
    with pytest.raises(ValueError, match="K"):
        b.s2o_evict(k, k, w, b.make_evict_params(1, 2, 128, 1000, 100))
    with pytest.raises(ValueError, match="both"):
        b.s2o_evict(k, None, w, b.make_evict_params(1, 2, 128, 1000, 100))


class _Tensor:
    """As much of a CUDA tensor as the layout check looks at."""
    is_cuda, device = True, torch.device("cuda:0")

    def __init__(self, shape, stride, dtype=torch.bfloat16):
        self.shape, self._stride, self.dtype = torch.Size(shape), tuple(stride), dtype

    def stride(self):
        return self._stride

    def is_contiguous(self):
        return self._stride == torch.empty(self.shape, device="meta").stride()


@pytest.mark.parametrize("shape,stride,kw", [
    ((1, 2, 5, 64), (640, 320, 64, 1), dict(dtype=torch.float16)),
    ((1, 2, 5, 64), (640, 320, 64, 1), dict(device=torch.device("cuda:1"))),
    ((1, 2, 4, 64), (640, 320, 64, 1), {}),
    ((1, 2, 5, 64), (640, 64, 128, 1), {}),
    ((1, 2, 5, 64), (640, 320, 64, 1), dict(strides=(640, 64, 128))),
    ((1, 2, 5, 64), (640, 64, 128, 2), dict(strides=(640, 64, 128))),
])
def test_layout_check_refuses(shape, stride, kw):
    t = _Tensor(shape, stride, kw.get("dtype", torch.bfloat16))
    with pytest.raises(ValueError):
        b._check_layout("K", t, torch.bfloat16, kw.get("device", t.device), (1, 2, 5, 64), kw.get("strides"))


def test_layout_check_takes_what_it_should():
    b._check_layout("K", _Tensor((1, 2, 5, 64), (640, 320, 64, 1)), torch.bfloat16, _Tensor.device, (1, 2, 5, 64))
    b._check_layout("K", _Tensor((1, 2, 5, 64), (7, 64, 128, 1)), torch.bfloat16, _Tensor.device, (1, 2, 5, 64), (640, 64, 128))


def test_layouts_follow_a_changed_struct():
    """A parameter struct is read by value at every call, not remembered by identity."""
    p = b.make_decode_params(1, 2, 4, 2, 128, 1, 1000)
    assert b._decode_layout(bytes(p))[0]["K"][0] == (1, 2, 1000, 128)
    p.cache_len = 77
    assert b._decode_layout(bytes(p))[0]["K"][0] == (1, 2, 77, 128)
    p.dtype = b.S2O_F16
    assert b._decode_layout(bytes(p))[1] is torch.float16


def test_bad_names_of_types_and_strides():
    with pytest.raises(ValueError, match="dtype"):
        b.make_evict_params(1, 1, 64, 10, 5, dtype="f32")
    with pytest.raises(ValueError, match="strides"):
        b.make_evict_params(1, 1, 64, 10, 5, k_stride=(640, 64))


def test_other_device_and_stream(monkeypatch):
    """A call goes to the tensors' device: its own current stream where none is given; a stream of another device is refused."""
    class _S:
        def __init__(self, device, handle):
            self.device, self.cuda_stream = torch.device(device), handle
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: _S(d, 0x70))
    handle, ctx = b._on_device(torch.device("cuda:1"), None)
    assert handle == 0x70 and isinstance(ctx, torch.cuda.device)
    assert b._on_device(torch.device("cuda:0"), _S("cuda:0", 0x80)) == (0x80, None)
    with pytest.raises(ValueError, match="stream"):
        b._on_device(torch.device("cuda:0"), _S("cuda:1", 0x80))


# ---- outputs and scratch on top of something else
def _spread(n):
    return [C.c_void_p((i + 1) << 28) for i in range(n)]


def test_decode_refuses_overlaps(lib):
    p = b.make_decode_params(2, 3, 4, 2, 128, 1, 5000, 10)
    at = _spread(10)
    need = b.s2o_decode_sizes(p)["scratch"]
    args = at[:7] + [C.byref(p), at[7], at[8], at[9], need, None]
    cases = [(8, at[i], b.S2O_EINVAL) for i in range(7)] + [(9, at[i], b.S2O_EINVAL) for i in range(8)] + [(10, at[i], b.S2O_EINVAL) for i in range(9)]
    q = 2 * 3 * 4 * 128 * 2                                                          # the last bytes of Q, of O, of K
    cases += [(8, C.c_void_p(at[0].value + q - 16), b.S2O_EINVAL), (9, C.c_void_p(at[7].value + q - 4), b.S2O_EINVAL),
              (8, C.c_void_p(at[1].value + 2 * 2 * 5000 * 256 - 16), b.S2O_EINVAL), (10, C.c_void_p(at[8].value - 256), b.S2O_EINVAL)]
    _refused(lib.s2o_decode, args, cases)


def test_weights_refuse_overlaps(lib):
    p = b.make_weights_params(1, 1, 4, 2, 128, 64, 10000, causal=1)
    at = _spread(7)
    need = b.s2o_key_weights_sizes(p)["scratch"]
    # Q K lse lens params prev weights scratch
    args = at[:4] + [C.byref(p), at[4], at[5], at[6], need, None]
    _refused(lib.s2o_key_weights, args, [(6, at[i], b.S2O_EINVAL) for i in range(4)] + [(6, C.c_void_p(at[4].value + 4), b.S2O_EINVAL)])
    args[2] = None                                                                   # (it needs scratch then)
    _refused(lib.s2o_key_weights, args, [(7, at[i], b.S2O_EINVAL) for i in (0, 1, 3, 4, 5)] + [(6, C.c_void_p(at[6].value + need - 4), b.S2O_EINVAL)])


def test_evict_refuses_scratch_on_top_of_an_output(lib):
    p = b.make_evict_params(1, 2, 128, 100000, 100)
    at = _spread(10)
    need = b.s2o_evict_sizes(p)["scratch"]
    args = at[:4] + [C.byref(p)] + at[4:9] + [at[9], need, None]
    _refused(lib.s2o_evict, args, [(10, x, b.S2O_EINVAL) for x in at[:9]])


def test_launches_that_do_not_fit_are_refused(lib):
    at = [C.c_void_p((i + 1) << 46) for i in range(10)]
    p = b.make_decode_params(1, 1 << 24, 4, 4, 128, 1, 96, 24)
    assert lib.s2o_decode(*at[:7], C.byref(p), at[7], at[8], at[9], 1 << 62, None) == b.S2O_EUNSUPPORTED
    p = b.make_decode_params(1 << 22, 64, 4, 4, 64, 1, 1000)
    assert lib.s2o_decode(*at[:3], None, None, None, None, C.byref(p), at[7], at[8], at[9], 1 << 62, None) == b.S2O_EUNSUPPORTED
    p = b.make_weights_params(1 << 23, 1, 2, 2, 64, 1, 70)
    assert lib.s2o_key_weights(at[0], at[1], at[2], None, C.byref(p), None, at[3], None, 0, None) == b.S2O_EUNSUPPORTED
    assert lib.s2o_key_weights(at[0], at[1], None, None, C.byref(p), None, at[3], at[4], 1 << 62, None) == b.S2O_EUNSUPPORTED
    p = b.make_evict_params(1 << 23, 2, 64, 100, 10)
    assert lib.s2o_evict(at[0], at[1], at[2], None, C.byref(p), at[3], at[4], None, at[5], None, None, 0, None) == b.S2O_EUNSUPPORTED
