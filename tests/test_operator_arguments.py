"""What the operators around the cache refuse, and what they compute on the host: checked without a GPU.  Arguments are
looked at before the handle or any buffer is, so a block of zeros stands for a handle and numbers stand for addresses."""
import ctypes
import math

import pytest

from paper_2511_16786_b200 import binding as fc

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
A = 1 << 20                                            # an aligned address that nothing reads


@pytest.fixture(scope="module")
def handle():
    return ctypes.create_string_buffer(1 << 16)


def _changed(make, call, **kw):
    a = make()
    for k, v in kw.items():
        setattr(a, k, v)
    return call(a)


# ---------------------------------------------------------------------------------------------- rotary
def _rotary():
    table = (ctypes.c_double * 64)(*([1.0] * 64))
    a = fc.fc_rotary_args(q=A, out_q=A, q_stride_token=512, q_stride_head=128, out_q_stride_token=512, out_q_stride_head=128,
                          k=A, out_k=A, k_stride_token=128, k_stride_head=128, out_k_stride_token=128, out_k_stride_head=128,
                          positions=A, position_stride=0, tokens=0, scale=1.0, dtype=fc.FC_BF16, num_q_heads=4, num_heads=1,
                          head_dim=128, rotary_dim=128)
    a.freq = ctypes.cast(table, ctypes.POINTER(ctypes.c_double))
    a._kept = table
    return a


def test_rotary_refusals(handle):
    def call(a):
        return fc._lib.fc_rotary(handle, ctypes.byref(a), None)

    assert call(_rotary()) == OK                       # no tokens: nothing to do, nothing launched
    assert fc._lib.fc_rotary(None, ctypes.byref(_rotary()), None) == INVALID
    assert fc._lib.fc_rotary(handle, None, None) == INVALID
    for kw in (dict(positions=None), dict(tokens=-1), dict(q=None, k=None), dict(out_q=None), dict(out_k=None), dict(num_q_heads=0),
               dict(num_heads=0), dict(v=A), dict(out_v=A), dict(q=A + 2), dict(out_k=A + 8), dict(q_stride_token=4),
               dict(out_k_stride_head=100), dict(v=A + 4, out_v=A), dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=130),
               dict(scale=math.inf), dict(scale=math.nan), dict(sections=(ctypes.c_int32 * 3)(16, 24, 25)),
               dict(sections=(ctypes.c_int32 * 3)(-1, 41, 24)), dict(out_rows=A, out_capacity_rows=-1),
               dict(out_rows=A, k=None, out_k=None), dict(k=None, v=A, out_v=A)):
        assert _changed(_rotary, call, **kw) == INVALID, kw
    for kw in (dict(dtype=3), dict(dtype=-1), dict(head_dim=96), dict(head_dim=0), dict(head_dim=1088, rotary_dim=64),
               dict(head_dim=512, rotary_dim=512), dict(num_q_heads=5000), dict(tokens=1 << 31)):
        assert _changed(_rotary, call, **kw) == UNSUPPORTED, kw
    for bad in (math.inf, -math.inf, math.nan):
        a = _rotary()
        a._kept[63] = bad
        assert call(a) == INVALID
    a = _rotary()
    a.freq = None
    assert call(a) == INVALID
    assert _changed(_rotary, call, sections=(ctypes.c_int32 * 3)(16, 24, 24)) == OK


def test_rotary_frequencies():
    f, scale = fc.fc_rotary_frequencies(128, 1e6)
    assert len(f) == 64 and scale == 1.0
    for j in (0, 1, 31, 63):
        assert f[j] == pytest.approx(1e6 ** (-j / 64), rel=1e-13)
    lin, scale = fc.fc_rotary_frequencies(128, 1e6, "linear", 4.0)
    assert scale == 1.0 and all(a == pytest.approx(b / 4, rel=1e-14) for a, b in zip(lin, f))
    # ntk: the first pair keeps its frequency, the last one gets exactly 1 / factor of it
    ntk, scale = fc.fc_rotary_frequencies(128, 1e4, "ntk", 8.0)
    plain, _ = fc.fc_rotary_frequencies(128, 1e4)
    assert ntk[0] == 1.0 and ntk[63] == pytest.approx(plain[63] / 8.0, rel=1e-12)
    # yarn and bands: many turns over the original length keep, few are divided by the factor, monotone in between
    for kind in ("yarn", "bands"):
        y, scale = fc.fc_rotary_frequencies(128, 1e4, kind, 4.0, 4096)
        assert scale == pytest.approx(0.1 * math.log(4.0) + 1.0 if kind == "yarn" else 1.0)
        share = [a / b for a, b in zip(y, plain)]
        assert share[0] == 1.0 and share[-1] == pytest.approx(0.25)
        assert all(a >= b - 1e-12 for a, b in zip(share, share[1:]))
        for j, x in enumerate(plain):
            turns = 4096 * x / (2 * math.pi)
            if turns > 40.0:
                assert share[j] == 1.0
            if turns < 0.9:
                assert share[j] == pytest.approx(0.25)
    turns = [4096 * x / (2 * math.pi) for x in plain]
    y, _ = fc.fc_rotary_frequencies(128, 1e4, "bands", 4.0, 4096)
    j = next(i for i, t in enumerate(turns) if 1.0 < t < 4.0)
    m = (turns[j] - 1.0) / 3.0
    assert y[j] == pytest.approx(plain[j] * (m + (1 - m) / 4.0), rel=1e-12)
    # factor 1 changes nothing
    for kind in ("linear", "ntk", "yarn", "bands"):
        one, scale = fc.fc_rotary_frequencies(64, 5e5, kind, 1.0, 8192)
        assert scale == 1.0 and one == pytest.approx(fc.fc_rotary_frequencies(64, 5e5)[0], rel=1e-14)


@pytest.mark.parametrize("args", [(0, 1e4), (3, 1e4), (258, 1e4), (128, 1.0), (128, math.inf), (128, math.nan), (128, 1e4, "linear", 0.5),
                                  (128, 1e4, "linear", math.inf), (128, 1e4, "yarn", 4.0, 0), (128, 1e4, "bands", 4.0, 4096, 4.0, 4.0),
                                  (128, 1e4, "yarn", 4.0, 4096, 0.0, 32.0), (2, 1e4, "ntk", 2.0), (128, 1e4, "linear", math.nan)])
def test_rotary_frequencies_refusals(args):
    with pytest.raises(fc.FlashCacheError) as e:
        fc.fc_rotary_frequencies(*args)
    assert e.value.code == INVALID
    with pytest.raises(ValueError):
        fc.fc_rotary_frequencies(128, 1e4, "other")


# ---------------------------------------------------------------------------------------------- 4-bit caches
def _cache():
    return fc.fc_cache4(A, A, A, A, 64, fc.FC_BF16, 2, 128)


_CACHE_REFUSALS = [(dict(codes_k=None), INVALID), (dict(codes_v=None), INVALID), (dict(params_k=None), INVALID),
                   (dict(params_v=None), INVALID), (dict(codes_k=A + 8), INVALID), (dict(params_v=A + 8), INVALID),
                   (dict(capacity_rows=0), INVALID), (dict(capacity_rows=24), INVALID), (dict(capacity_rows=-16), INVALID),
                   (dict(num_heads=0), INVALID), (dict(dtype=fc.FC_F32), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
                   (dict(head_dim=96), UNSUPPORTED), (dict(capacity_rows=1 << 31), UNSUPPORTED), (dict(num_heads=1 << 17), UNSUPPORTED)]


def test_cache4_refusals(handle):
    cu = (ctypes.c_int32 * 2)(0, 0)

    def view(**kw):
        v = fc.fc_kv_view(A, A, 256, 128, fc.FC_BF16, 2, 128, 1, ctypes.cast(cu, ctypes.POINTER(ctypes.c_int32)))
        for k, x in kw.items():
            setattr(v, k, x)
        return v

    def quantize(c, v, rows=None):
        return fc._lib.fc_quantize_cache(handle, ctypes.byref(v), ctypes.byref(c), None, rows, None)

    def back(c, rows=0, k=A, v=A):
        return fc._lib.fc_dequantize_cache(handle, ctypes.byref(c), k, v, rows, None, None)

    assert quantize(_cache(), view()) == OK and back(_cache()) == OK      # no rows
    for kw, want in _CACHE_REFUSALS:
        c = _cache()
        for k, x in kw.items():
            setattr(c, k, x)
        assert quantize(c, view()) == want and back(c) == want, kw
    for kw in (dict(k=None), dict(v=None), dict(cu_seqlens=None), dict(batch=0), dict(dtype=fc.FC_F16), dict(num_heads=1),
               dict(head_dim=64), dict(k=A + 8), dict(stride_token=4), dict(stride_head=12)):
        assert quantize(_cache(), view(**kw)) == INVALID, kw
    cu[1] = 65                                          # more rows than the cache has
    assert quantize(_cache(), view()) == INVALID
    cu[1] = -1
    assert quantize(_cache(), view()) == INVALID
    assert back(_cache(), 65) == INVALID and back(_cache(), -1) == INVALID
    assert back(_cache(), 1, None) == INVALID and back(_cache(), 1, A, A + 8) == INVALID
    for args in ((None, ctypes.byref(view()), ctypes.byref(_cache())), (handle, None, ctypes.byref(_cache())),
                 (handle, ctypes.byref(view()), None)):
        assert fc._lib.fc_quantize_cache(*args, None, None, None) == INVALID
    assert fc._lib.fc_dequantize_cache(None, ctypes.byref(_cache()), A, A, 0, None, None) == INVALID


def test_rows_past_the_last_int_are_refused(handle):
    cu, cache = (ctypes.c_int32 * 2)(0, (1 << 31) - 1), _cache()
    view = fc.fc_kv_view(A, A, 256, 128, fc.FC_BF16, 2, 128, 1, ctypes.cast(cu, ctypes.POINTER(ctypes.c_int32)))
    assert fc._lib.fc_quantize_cache(handle, ctypes.byref(view), ctypes.byref(cache), None, A, None) == UNSUPPORTED
    cu[1] = 65                                              # more than the cache has, without rows to go to
    assert fc._lib.fc_quantize_cache(handle, ctypes.byref(view), ctypes.byref(cache), None, None, None) == INVALID
