"""fc_quantize_cache and fc_dequantize_cache against their definition in 64 bits: codes, scales and minima are whole
decisions and have to be equal; a value is min + scale * code, exact in fp32 up to its last sum, rounded to the type."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DIGITS = {torch.bfloat16: (8, -133), torch.float16: (11, -24)}      # significant bits, smallest step


@pytest.fixture(scope="module")
def fc():
    from paper_2511_16786_b200 import binding
    return binding


@pytest.fixture(scope="module")
def handle(fc):
    h = fc.fc_create(0, 1024)
    yield h
    assert fc.fc_last_device_status(h) == 0
    fc.fc_destroy(h)


def _definition(x):
    """x [rows, H, d] of a 16-bit type -> codes [rows, H, d], scale and minimum [rows, H, 2] in 64 bits."""
    digits, least = DIGITS[x.dtype]
    y = x.double().cpu().numpy().reshape(x.shape[0], x.shape[1], 2, -1)
    lo, hi = y.min(-1), y.max(-1)
    want = (hi - lo) / 15
    unit = 2.0 ** np.maximum(np.frexp(want)[1] - digits, least)
    scale = np.ceil(want / unit) * unit
    t = np.divide(y - lo[..., None], scale[..., None], out=np.zeros_like(y), where=scale[..., None] > 0)
    codes = np.rint(t)                                  # half to even
    return codes.reshape(x.shape), scale, lo


def _nibbles(codes, dim, values):
    """Codes of a cache [H, rows, d/2] as [rows, H, d], by the order the header of the layout gives."""
    c = codes.cpu().numpy()
    nib = np.stack((c & 15, c >> 4), -1).reshape(c.shape[0], c.shape[1], dim)
    at = np.empty(dim, dtype=int)
    for ch in range(dim):
        if values:
            at[ch] = (ch % 8) * (dim // 8) + ch // 8
        else:
            s, t, i = ch // 16, ch // 4 % 4, ch % 4
            at[ch] = t * (dim // 4) + (s // 2) * 8 + (i % 2) * 4 + i // 2 + 2 * (s % 2)
    return nib[:, :, at].transpose(1, 0, 2)


def _check(cache, k, v, rows=None):
    n, H, d = k.shape
    rows = list(range(n)) if rows is None else rows
    for x, codes, params, values in ((k, cache.codes_k, cache.params_k, False), (v, cache.codes_v, cache.params_v, True)):
        want, scale, lo = _definition(x)
        p = params.double().cpu().numpy()[:, rows].transpose(1, 0, 2)
        np.testing.assert_array_equal(p[..., 0::2], scale)
        np.testing.assert_array_equal(p[..., 1::2], lo)
        np.testing.assert_array_equal(_nibbles(codes, d, values)[rows], want)


def _back(fc, handle, cache, n, dtype):
    out = [torch.full((n, cache.num_heads, cache.head_dim), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    fc.fc_dequantize_cache(handle, cache, *out)
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,H,d", [(1, 1, 64), (1, 1, 128), (17, 3, 64), (65, 5, 128), (4099, 2, 128), (2000, 7, 64)])
def test_quantized_rows_are_the_definitions(fc, handle, n, H, d, dtype):
    g = torch.Generator().manual_seed(n + H)
    k = (torch.randn((n, H, d), generator=g) * 3 + torch.randn((1, H, d), generator=g)).to(dtype).cuda()
    v = torch.randn((n, H, d), generator=g).to(dtype).cuda()
    cache = fc.Cache4.empty(n, H, d, dtype)
    for t in (cache.codes_k, cache.codes_v):
        t.fill_(0x5a)
    fc.fc_quantize_cache(handle, k, v, cache)
    _check(cache, k, v)
    for x, out in zip((k, v), _back(fc, handle, cache, n, dtype)):
        codes, scale, lo = _definition(x)
        half = codes.reshape(n, H, 2, -1)
        exact = lo[..., None] + scale[..., None] * half
        got = out.double().cpu().numpy().reshape(exact.shape)
        assert (np.abs(got - exact) <= torch.finfo(dtype).eps / 2 * np.abs(exact) * (1 + 1e-6) + 2.0 ** -24 * np.abs(lo[..., None])).all()
        # no value moved by more than half a step, beside the rounding of the value itself
        moved = np.abs(exact - x.double().cpu().numpy().reshape(exact.shape))
        assert (moved <= scale[..., None] / 2).all()
    assert (cache.codes_k[:, n:] == 0x5a).all() and (cache.codes_v[:, n:] == 0x5a).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_quantizing_at_the_edges_of_the_numbers(fc, handle, dtype):
    d = 64
    tiny = DIGITS[dtype][1]
    big = float(torch.finfo(dtype).max)
    rows = [torch.zeros(d), torch.full((d,), -3.25), torch.arange(d) / 4.0, -torch.arange(d).float(),
            torch.arange(d) * 2.0 ** tiny,                                        # subnormal steps
            torch.arange(d) * 2.0 ** (tiny + 3) - 2.0 ** (tiny + 8),
            (torch.arange(d) % 16).float(),                                       # codes themselves
            (torch.arange(d) % 31) * 0.5,                                         # every second value is a tie
            (torch.arange(d) % 31) * -0.5 + 7.5,
            torch.where(torch.arange(d) % 2 == 0, -7.5, 7.5).index_fill(0, torch.tensor([5]), 2.0 ** (tiny + 2)),   # beside a tie
            torch.where(torch.arange(d) % 2 == 0, -7.5, 7.5).index_fill(0, torch.tensor([5, 37]), -(2.0 ** (tiny + 2))),
            torch.where(torch.arange(d) % 3 == 0, -big / 4, big / 4),
            torch.where(torch.arange(d) == 9, big / 2, 1.0),
            torch.linspace(-1, 1, d) * 2.0 ** -20, torch.linspace(100.0, 100.5, d)]
    k = torch.stack(rows).to(dtype).view(len(rows), 1, d).cuda()
    v = torch.flip(k, (0, 2)).contiguous()
    cache = fc.Cache4.empty(len(rows), 1, d, dtype)
    fc.fc_quantize_cache(handle, k, v, cache)
    _check(cache, k, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_pair_of_a_small_range_is_decided_exactly(fc, handle, dtype):
    # values on a coarse grid against scales on another one: thousands of quotients at or beside a half
    g = torch.Generator().manual_seed(11)
    x = torch.randint(-40, 41, (3000, 2, 128), generator=g).float() * 0.25
    x = x * 2.0 ** torch.randint(-3, 4, (3000, 2, 1), generator=g)
    k, v = x.to(dtype).cuda(), x.flip(2).to(dtype).cuda()
    cache = fc.Cache4.empty(3000, 2, 128, dtype)
    fc.fc_quantize_cache(handle, k, v, cache)
    _check(cache, k, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
def test_halves_that_are_not_finite_stand_for_nan(fc, handle, d, dtype):
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((6, 2, d), generator=g).to(dtype).cuda() for _ in range(2))
    k[1, 0, 3], k[2, 1, d - 1], v[3, 0, 0] = float("nan"), float("inf"), -float("inf")
    v[4, 1, d // 2], v[4, 1, d // 2 + 1] = float("inf"), -float("inf")
    cache = fc.Cache4.empty(6, 2, d, dtype)
    fc.fc_quantize_cache(handle, k, v, cache)
    for x, out in zip((k, v), _back(fc, handle, cache, 6, dtype)):
        bad = ~torch.isfinite(x.view(6, 2, 2, -1)).all(-1, keepdim=True).expand(-1, -1, -1, d // 2).reshape(x.shape)
        assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()
    # halves beside them are what they would be alone
    clean_k, clean_v = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
    other = fc.Cache4.empty(6, 2, d, dtype)
    fc.fc_quantize_cache(handle, clean_k, clean_v, other)
    a, b = _back(fc, handle, cache, 6, dtype)[0], _back(fc, handle, other, 6, dtype)[0]
    assert torch.equal(a[torch.isfinite(a)], b[torch.isfinite(a)])


def test_bf16_range_past_fp32_stands_for_nan(fc, handle):
    x = torch.full((1, 1, 64), 1.0, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 0], x[0, 0, 1] = 3e38, -3e38
    cache = fc.Cache4.empty(1, 1, 64, torch.bfloat16)
    fc.fc_quantize_cache(handle, x, x, cache)
    out = _back(fc, handle, cache, 1, torch.bfloat16)[0]
    assert torch.isnan(out[0, 0, :32]).all() and (out[0, 0, 32:] == 1).all()


@pytest.mark.parametrize("d", [64, 128])
def test_rows_go_where_they_are_sent_and_only_the_used_ones(fc, handle, d):
    n, H = 70, 3
    g = torch.Generator().manual_seed(7)
    wide = torch.randn((n, H, d + 64), generator=g).to(torch.bfloat16).cuda()
    k, v = wide[:, :, :d], torch.randn((n, H, d + 64), generator=g).to(torch.bfloat16).cuda()[:, :, :d]      # rows apart
    cache = fc.Cache4.empty(100, H, d, torch.bfloat16)
    for t in (cache.codes_k, cache.codes_v):
        t.fill_(0xee)
    for t in (cache.params_k, cache.params_v):
        t.fill_(5.0)
    to = torch.randperm(cache.capacity_rows, generator=g)[:n].cuda()
    to[4] = -1
    used = torch.tensor([50], device="cuda")
    fc.fc_quantize_cache(handle, k, v, cache, used=used, out_rows=to)
    took = [i for i in range(50) if i != 4]
    _check(cache, k[took], v[took], [int(to[i]) for i in took])
    rest = sorted(set(range(cache.capacity_rows)) - {int(to[i]) for i in took})
    assert (cache.codes_k[:, rest] == 0xee).all() and (cache.codes_v[:, rest] == 0xee).all()
    assert (cache.params_k[:, rest] == 5).all() and (cache.params_v[:, rest] == 5).all()
    assert fc.fc_last_device_status(handle) == 0
    to[9] = cache.capacity_rows                          # behind the cache: left out and said
    fc.fc_quantize_cache(handle, k, v, cache, used=used, out_rows=to)
    assert fc.fc_last_device_status(handle) == 6
    # counts below zero and past the rows
    for count, first in ((-5, 0), (0, 0), (1000, n), (13, 13)):
        fresh = fc.Cache4.empty(100, H, d, torch.bfloat16)
        for t in (fresh.params_k, fresh.params_v):
            t.fill_(5.0)
        used.fill_(count)
        fc.fc_quantize_cache(handle, k, v, fresh, used=used)
        assert (fresh.params_k[:, first:] == 5).all() and (first == 0 or not (fresh.params_k[:, :first] == 5).all())
        out = [torch.full((n, H, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        fc.fc_dequantize_cache(handle, fresh, *out, used=used)
        assert (out[0][first:] == 9).all() and (out[1][first:] == 9).all()
        if first:
            assert not (out[0][:first] == 9).all()


def test_quantizing_captured_and_replayed_on_new_rows(fc, handle):
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((300, 2, 128), generator=g).to(torch.float16).cuda() for _ in range(2))
    cache = fc.Cache4.empty(300, 2, 128, torch.float16)
    used = torch.tensor([300], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fc.fc_quantize_cache(handle, k, v, cache, used=used)
    k.mul_(-2.0)
    graph.replay()
    torch.cuda.synchronize()
    _check(cache, k, v)


def test_cache_argument_checks_of_the_binding(fc):
    c = fc.Cache4.empty(20, 2, 64, torch.bfloat16)
    assert c.capacity_rows == 32 and c.nbytes == 2 * 2 * 32 * (32 + 8)
    with pytest.raises(ValueError):
        fc.Cache4(c.codes_k, c.codes_v[:, :16], c.params_k, c.params_v)
    with pytest.raises(ValueError):
        fc.Cache4(c.codes_k, c.codes_v, c.params_k, c.params_v.half())
    with pytest.raises(ValueError):
        fc.Cache4(c.codes_k, c.codes_v, c.params_k[:, :, :2], c.params_v)
    k = torch.zeros((20, 2, 64), dtype=torch.bfloat16, device="cuda")
    h = ctypes.create_string_buffer(1 << 16)
    with pytest.raises(ValueError):
        fc.fc_quantize_cache(h, k, k, c, used=torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        fc.fc_quantize_cache(h, k, k, c, out_rows=torch.zeros(19, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        fc.fc_dequantize_cache(h, c, k, k.half())
    with pytest.raises(fc.FlashCacheError):
        fc.fc_quantize_cache(h, k.half(), k.half(), c)


@pytest.mark.parametrize("used", [0, -1, 5 - 2 ** 32, 5 - 2 ** 63, 2 ** 32 + 5])
def test_counts_of_rows_outside_the_rows(fc, handle, used):
    """Negative ones name no row, ones past the rows all of them, however many bits they have."""
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((10, 3, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    cache = fc.Cache4.empty(10, 3, 64, torch.bfloat16)
    whole = [torch.empty_like(k), torch.empty_like(v)]
    fc.fc_quantize_cache(handle, k, v, cache)
    fc.fc_dequantize_cache(handle, cache, *whole)
    count = torch.tensor([used], device="cuda")
    outs = [torch.full_like(k, 7.0), torch.full_like(v, 7.0)]
    fc.fc_dequantize_cache(handle, cache, *outs, used=count)
    other = fc.Cache4.empty(10, 3, 64, torch.bfloat16)
    for t in (other.codes_k, other.codes_v, other.params_k, other.params_v):
        t.fill_(7)
    before = other.codes_k.clone()
    fc.fc_quantize_cache(handle, k, v, other, used=count)
    for out, all_of_them in zip(outs, whole):
        assert torch.equal(out, all_of_them if used > 0 else torch.full_like(out, 7.0))
    assert torch.equal(other.codes_k[:, :10], cache.codes_k[:, :10] if used > 0 else before[:, :10])
