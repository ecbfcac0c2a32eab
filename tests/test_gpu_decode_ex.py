"""fc_decode_attention_ex (4-bit rows, windows with sinks) against its definition in 64 bits.

Tolerance, derived element by element.  A weight beside a 4-bit row is rounded once to fp16 (2^-11 of it), beside a 16-bit
row to the type (eps / 2).  Scores are sums of d products in fp32, keys taken as minimum plus scale * code: each of the at
most d + 8 additions is off by 2^-23 (the tensor cores cut off) of the sum of the products' sizes, which moves every weight by
as much; twice, since the sum of the weights moves too.  Sums of weights and the rest: 2^-16.  Then half a step of the output's
type.  All of it times the mean of the values' sizes under the weights, a value's size being |minimum| + scale * code."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2511_16786_b200 import binding as fc

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def _order(dim, values):
    if values:
        return [(c % 8) * (dim // 8) + c // 8 for c in range(dim)]
    return [(c // 4 % 4) * (dim // 4) + (c // 32) * 8 + 4 * (c % 2) + c % 4 // 2 + 2 * (c // 16 % 2) for c in range(dim)]


def _held(codes, params, values):
    """A 4-bit cache as ([rows, H, d] values, [rows, H, d] sizes) in 64 bits."""
    c, p = codes.cpu().numpy(), params.double().cpu().numpy()
    dim = 2 * c.shape[2]
    nib = np.stack((c & 15, c >> 4), -1).reshape(c.shape[0], c.shape[1], dim)[:, :, _order(dim, values)]
    half = nib.reshape(*nib.shape[:2], 2, -1).astype(np.float64)
    with np.errstate(invalid="ignore"):                                    # rows nobody wrote
        low, step = p[..., 1::2, None], p[..., 0::2, None] * half
    return [x.reshape(nib.shape).transpose(1, 0, 2) for x in (low + step, np.abs(low) + step)]


def _definition(q, main, offsets, tail, tail_len, window, sinks, dtype, four):
    """-> (out, tolerance), [B, Hq, d].  main: (k, |k|, v, |v|) of the kept rows in 64 bits; tail: (k, v) or None."""
    q = q.double().cpu().numpy()
    B, Hq, d = q.shape
    H = main[0].shape[1]
    G = Hq // H
    out, tol = np.zeros_like(q), np.zeros_like(q)
    eps = torch.finfo(dtype).eps
    for b in range(B):
        lo, hi = offsets[b], offsets[b + 1]
        parts = [x[lo:hi] for x in main]
        unit = np.full(hi - lo, 2.0 ** -11 if four else eps / 2)
        if tail is not None and tail_len[b]:
            tk, tv = (x[b, :tail_len[b]].double().cpu().numpy() for x in tail)
            parts = [np.concatenate(p) for p in zip(parts, (tk, np.abs(tk), tv, np.abs(tv)))]
            unit = np.concatenate((unit, np.full(tail_len[b], eps / 2)))
        n = parts[0].shape[0]
        j = np.arange(n)
        seen = (j < sinks) | (j >= n - window) if window else j >= 0
        if not seen.any():
            continue
        for hq in range(Hq):
            k, ka, v, va = (p[seen, hq // G] for p in parts)
            s = k @ q[b, hq] / math.sqrt(d)
            off = (d + 8) * 2.0 ** -23 * (ka @ np.abs(q[b, hq])).max() / math.sqrt(d)
            w = np.exp(s - s.max())
            w /= w.sum()
            out[b, hq] = w @ v
            tol[b, hq] = (w * (unit[seen] + 2 * off + 2.0 ** -16)) @ va + eps / 2 * np.abs(out[b, hq]) + torch.finfo(dtype).smallest_normal
    return out, tol


@pytest.fixture(scope="module")
def handle():
    h = fc.fc_create(0, 1024)
    yield h
    assert fc.fc_last_device_status(h) == 0
    fc.fc_destroy(h)


def _case(lens, tails, H, G, d, dtype, four, handle, seed, spare=5, peaked=1.0, cap=80):
    g = torch.Generator().manual_seed(seed)
    B, rows = len(lens), max(sum(lens), 1) + spare
    offs = [int(x) for x in np.cumsum([0] + lens)]
    q = (torch.randn((B, H * G, d), generator=g) * peaked).to(dtype).cuda()
    k = (torch.randn((rows, H, d), generator=g) + torch.randn((1, H, d), generator=g)).to(dtype).cuda()
    v = (torch.randn((rows, H, d), generator=g) + 0.5).to(dtype).cuda()
    tail = None
    if tails:
        tail = [torch.randn((B, cap, H, d), generator=g).to(dtype).cuda() for _ in range(2)]
    if four:
        cache = fc.Cache4.empty(rows, H, d, dtype)
        for t in (cache.codes_k, cache.codes_v):
            t.fill_(0xff)
        for t in (cache.params_k, cache.params_v):
            t.fill_(float("nan"))
        fc.fc_quantize_cache(handle, k, v, cache)
        main = _held(cache.codes_k, cache.params_k, False) + _held(cache.codes_v, cache.params_v, True)
    else:
        cache = (k, v)
        kd, vd = k.double().cpu().numpy(), v.double().cpu().numpy()
        main = [kd, np.abs(kd), vd, np.abs(vd)]
    return q, cache, main, offs, tail


def _run(handle, q, cache, offs, tail, tails, window, sinks, most=None, times=1):
    B = q.shape[0]
    od = torch.tensor(offs, dtype=torch.int64, device="cuda")
    tl = torch.tensor(tails, dtype=torch.int32, device="cuda") if tails else None
    if most is None:
        most = max(offs[b + 1] - offs[b] + (tails[b] if tails else 0) for b in range(B))
    args, opt = fc.make_decode_args_ex(q, cache, od, most, tail[0] if tail else None, tail[1] if tail else None, tl, window, sinks)
    ws = torch.empty(fc.fc_decode_workspace_bytes_ex(handle, args, opt), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    for _ in range(times):
        fc.fc_decode_attention_ex(handle, args, opt, out, ws)
    assert fc.fc_last_device_status(handle) == 0
    return out


def _check(out, want, tol):
    got, undefined = out.double().cpu().numpy(), np.isnan(want)          # a value that stands for NaN, and only such, gives NaN
    np.testing.assert_array_equal(np.isnan(got), undefined)
    err = np.abs(got - want)[~undefined]
    assert (err <= tol[~undefined]).all(), "worst error / tolerance %.3f" % (err / np.maximum(tol[~undefined], 1e-300)).max()


SHAPES = [([1], None, 1, 1, 0, 0), ([127, 128, 129, 0, 1], None, 2, 7, 0, 0), ([0, 0, 5], [3, 0, 64], 3, 9, 0, 0),
          ([0, 300, 1, 4097], [1, 65, 0, 80], 4, 8, 0, 0), ([9601], None, 1, 16, 0, 0),
          ([333, 127] * 37, None, 2, 2, 0, 0), ([130, 70], [0, 5], 160, 1, 0, 0),
          # windows: within the kept rows, across into the tail, within the tail, longer than all, one row, no sinks, sinks past a tile
          ([700, 129, 1], [0, 33, 80], 2, 4, 100, 4), ([40, 0, 3], [50, 80, 2], 1, 7, 30, 10), ([1000, 5], [10, 0], 2, 8, 5000, 3),
          ([513, 1025, 77], None, 2, 12, 1, 0), ([2000, 301], [3, 7], 1, 4, 257, 200), ([5, 0], [70, 75], 2, 3, 20, 40),
          ([64 * 40], [32], 1, 1, 64, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("lens,tails,H,G,window,sinks", SHAPES)
def test_decode_ex_matches_the_definition(handle, lens, tails, H, G, window, sinks, four, d, dtype):
    q, cache, main, offs, tail = _case(lens, tails, H, G, d, dtype, four, handle, sum(lens) + d + G)
    out = _run(handle, q, cache, offs, tail, tails, window, sinks, times=2)
    want, tol = _definition(q, main, offs, tail, tails, window, sinks, dtype, four)
    _check(out, want, tol)
    for b, n in enumerate(lens):
        if n + (tails[b] if tails else 0) == 0:
            assert not out[b].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_what_has_no_weight_may_hold_anything(handle, four, window, sinks, dtype):
    lens, tails, H, G, d = [70, 1, 131, 400], [5, 0, 33, 70], 2, 4, 128
    q, cache, main, offs, tail = _case(lens, tails, H, G, d, dtype, four, handle, 77, spare=90)
    want, tol = _definition(q, main, offs, tail, tails, window, sinks, dtype, four)
    poison = [float("nan"), float("inf"), -float("inf")]
    hidden = list(range(offs[-1], offs[-1] + 90))
    for b, n in enumerate(lens):
        total = n + tails[b]
        hidden += [offs[b] + j for j in range(n) if window and sinks <= j < total - window]
        late = [j for j in range(80) if j >= tails[b] or (window and sinks <= n + j < total - window)]
        for i, j in enumerate(late):
            tail[0][b, j], tail[1][b, j] = poison[i % 3], poison[(i + 1) % 3]
    for i, r in enumerate(hidden):
        if four:
            cache.params_k[:, r], cache.params_v[:, r] = poison[i % 3], poison[(i + 1) % 3]
        else:
            cache[0][r], cache[1][r] = poison[i % 3], poison[(i + 1) % 3]
    _check(_run(handle, q, cache, offs, tail, tails, window, sinks), want, tol)
    # and a row that has weight does reach the output, of its own head and sequence only
    r = offs[3] + 1                                        # a sink where there is a window (row 399 would be outside it: 470 - 50 = 420)
    if four:
        cache.params_v[1, r, 1] = float("nan")
    else:
        cache[1][r, 1, :d // 2] = float("nan")
    out = _run(handle, q, cache, offs, tail, tails, window, sinks)
    assert torch.isnan(out[3, G:, :d // 2]).all()
    out[3, G:, :d // 2] = 0
    assert torch.isfinite(out).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size_k,size_v,peaked", [(1.0, 1.0, 6.0), (2.0 ** -9, 2.0 ** -9, 1.0), (1.0, 2.0 ** 9, 2.0), (2.0 ** -20, 2.0 ** -20, 2.0 ** 12),
                                                 (2.0 ** 30, 2.0 ** 40, 2.0 ** -28), (2.0 ** -60, 2.0 ** -36, 2.0 ** 55)])
def test_weights_and_values_of_unlike_sizes(handle, size_k, size_v, peaked, dtype):
    if dtype == torch.float16 and not (2.0 ** -10 < size_v < 2.0 ** 10 and size_k >= 2.0 ** -10 and peaked < 2.0 ** 10):
        size_k, size_v, peaked = min(max(size_k, 2.0 ** -4), 2.0 ** 5), min(max(size_v, 2.0 ** -6), 2.0 ** 11), min(max(peaked, 2.0 ** -5), 2.0 ** 4)
    g = torch.Generator().manual_seed(3)
    lens, H, G, d = [901, 2048], 2, 7, 128
    rows = sum(lens)
    q = (torch.randn((2, H * G, d), generator=g) * peaked).to(dtype).cuda()
    grow = 2.0 ** (torch.arange(rows) * 8 // rows).float()[:, None, None]            # values grow from row to row, keys do not
    k = (torch.randn((rows, H, d), generator=g) * size_k).to(dtype).cuda()
    v = (torch.randn((rows, H, d), generator=g) * size_v * grow / 16).to(dtype).cuda()
    cache = fc.Cache4.empty(rows, H, d, dtype)
    fc.fc_quantize_cache(handle, k, v, cache)
    main = _held(cache.codes_k, cache.params_k, False) + _held(cache.codes_v, cache.params_v, True)
    offs = [0, lens[0], rows]
    want, tol = _definition(q, main, offs, None, None, 0, 0, dtype, True)
    _check(_run(handle, q, cache, offs, None, None, 0, 0), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("most", [1, 128 * 40])
def test_scales_at_both_ends_of_bf16(handle, most, apart):
    """Rows of equal weight whose values are 2^165 apart: what a row adds to the sum of weights counts, however small its scale."""
    n, d = 128 * 40, 128
    g = torch.Generator().manual_seed(6)
    size = torch.full((n, 1, 1), 1e-13)
    size[torch.arange(n) >= n // 2 if apart else torch.arange(n) % 64 >= 32] = 8e37
    k, v = torch.zeros((n, 1, d), dtype=torch.bfloat16).cuda(), ((torch.rand((n, 1, d), generator=g) * 2 - 1) * size).to(torch.bfloat16).cuda()
    q = torch.randn((1, 4, d), generator=g).to(torch.bfloat16).cuda()
    cache = fc.Cache4.empty(n, 1, d, torch.bfloat16)
    fc.fc_quantize_cache(handle, k, v, cache)
    main = _held(cache.codes_k, cache.params_k, False) + _held(cache.codes_v, cache.params_v, True)
    want, tol = _definition(q, main, [0, n], None, None, 0, 0, torch.bfloat16, True)
    _check(_run(handle, q, cache, [0, n], None, None, 0, 0, most=most), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 12])
@pytest.mark.parametrize("large,far,tails", [(2.0 ** 30, 80.0, None), (2.0 ** 60, 80.0, None), (2.0 ** 60, 80.0, [70]), (2.0 ** 100, 110.0, None),
                                             (2.0 ** 40, 0.0, None)])
def test_rows_of_unlike_scales_hold_nothing_down(handle, large, far, tails, G, d):
    """Some rows' values are `large` times the others', and their weights 2^-far times those, before, between and after the others
    in every warp's rows; the odd query heads see it the other way round.  Values that small beside the large ones count."""
    n, H, g = 128 * 9 + 77, 2, torch.Generator().manual_seed(int(far) + d)
    rare = (torch.arange(n) // 8 % 3 == 0)
    base = torch.randn((H, 1, d), generator=g)
    q = (base * torch.tensor([1.0, -1.0]).repeat(G // 2)[:, None] + 0.05 * torch.randn((H, G, d), generator=g)).reshape(1, H * G, d)
    k, v = 0.2 * torch.randn((n, H, d), generator=g), torch.randn((n, H, d), generator=g)
    k[rare] -= (base / (base * base).sum(-1, keepdim=True) * far * math.sqrt(d) * math.log(2.0))[:, 0]
    v[rare] *= large
    q, k, v = (x.to(torch.bfloat16).cuda() for x in (q, k, v))
    tail = [torch.randn((1, 80, H, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2)] if tails else None
    cache = fc.Cache4.empty(n, H, d, torch.bfloat16)
    fc.fc_quantize_cache(handle, k, v, cache)
    main = _held(cache.codes_k, cache.params_k, False) + _held(cache.codes_v, cache.params_v, True)
    want, tol = _definition(q, main, [0, n], tail, tails, 0, 0, torch.bfloat16, True)
    for most in (1, n):                                                    # few blocks, and many
        _check(_run(handle, q, cache, [0, n], tail, tails, 0, 0, most=most), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size,other", [(2.0 ** 40, 1.0), (2.0 ** -100, 1.0), (2.0 ** -100, 2.0 ** -100), (2.0 ** 120, 2.0 ** -90)])
def test_halves_of_unlike_scales(handle, size, other, d):
    """The halves of a row are held with scales of their own, and neither costs the other bits."""
    lens, H, G = [700, 129], 2, 7
    g = torch.Generator().manual_seed(17)
    n = sum(lens)
    q, k = (torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((2, H * G, d), (n, H, d)))
    v = torch.randn((n, H, d), generator=g) + 0.5
    v[:, 0, :d // 2] *= size
    v[:, 1, d // 2:] *= size
    v[:, 0, d // 2:] *= other
    v[:, 1, :d // 2] *= other
    cache = fc.Cache4.empty(n, H, d, torch.bfloat16)
    fc.fc_quantize_cache(handle, k, v.to(torch.bfloat16).cuda(), cache)
    main = _held(cache.codes_k, cache.params_k, False) + _held(cache.codes_v, cache.params_v, True)
    want, tol = _definition(q, main, [0, 700, n], None, None, 0, 0, torch.bfloat16, True)
    _check(_run(handle, q, cache, [0, 700, n], None, None, 0, 0), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,G,tails", [(64, 1, None), (128, 7, None), (128, 12, [40])])
def test_a_row_with_all_the_weight_is_given_back(handle, d, G, tails, dtype):
    """The largest weight * scale is exact where a reference has just moved to it, so the output is the row's value, off by sums in
    fp32 (2^-16 of |minimum| + scale * code) and the rounding to the type; the other rows have 2^-60 of the weight."""
    lens, H, g = [300, 1], 2, torch.Generator().manual_seed(d + G)
    n = sum(lens)
    q, k, v = (torch.randn(s, generator=g) for s in ((2, H * G, d), (n, H, d), (n, H, d)))
    base = torch.randn(d, generator=g)
    q, k = base + 0.02 * q, 0.02 * k
    k[77] += base / (base @ base) * 60.0 * math.sqrt(d) * math.log(2.0)
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    cache = fc.Cache4.empty(n, H, d, dtype)
    fc.fc_quantize_cache(handle, k, v, cache)
    held, size = _held(cache.codes_v, cache.params_v, True)
    tail = [0.02 * torch.randn((2, 80, H, d), generator=g).to(dtype).cuda() for _ in range(2)] if tails else None
    out = _run(handle, q, cache, [0, 300, n], tail, tails + [0] if tails else None, 0, 0).double().cpu().numpy()
    for b, r in ((0, 77), (1, 300)):
        want, s = (np.repeat(x[r], G, 0) for x in (held, size))
        assert (np.abs(out[b] - want) <= torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -16 * s + torch.finfo(dtype).smallest_normal).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scores_that_are_all_minus_infinity_are_undefined(handle, dtype):
    """0 / 0 by the definition, for the queries and sequences that see nothing else."""
    lens, H, G, d = [40, 300, 2], 2, 4, 64
    q, (k, v), main, offs, _ = _case(lens, None, H, G, d, dtype, False, handle, 8)
    q.abs_().add_(0.5)
    k[40:340, 1] = float("-inf")
    k[340, 0] = float("-inf")
    got = _run(handle, q, (k, v), offs, None, None, 0, 0).isnan()
    want = torch.zeros_like(got)
    want[1, G:] = True
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_bound_of_rows_changes_the_launch_only_and_rows_past_the_cache_are_none(handle):
    lens, H, G, d = [500, 64, 3001], 2, 7, 128
    q, cache, main, offs, tail = _case(lens, None, H, G, d, torch.bfloat16, True, handle, 5)
    want, tol = _definition(q, main, offs, None, None, 0, 0, torch.bfloat16, True)
    for most in (3001, 50000, 1):
        _check(_run(handle, q, cache, offs, None, None, 0, 0, most=most), want, tol)
    # offsets that pass the cache's end, or run backwards, name no rows there
    far = [0, 500, 564, cache.capacity_rows + 1000]
    main_far = [x[:cache.capacity_rows] for x in main]
    cache.params_k[:, offs[-1]:], cache.params_v[:, offs[-1]:] = 0.0, 0.0
    for x in main_far:
        x[offs[-1]:] = 0.0
    want, tol = _definition(q, main_far, [0, 500, 564, cache.capacity_rows], None, None, 0, 0, torch.bfloat16, True)
    _check(_run(handle, q, cache, far, None, None, 0, 0, most=4000), want, tol)
    out = _run(handle, q, cache, [0, 500, 100, 50], None, None, 0, 0, most=4000)
    assert not out[1:].any()


@pytest.mark.gpu
def test_options_null_is_the_plain_call_and_16_bit_rows_agree_with_it(handle):
    lens, tails, H, G, d = [700, 33], [9, 64], 4, 7, 128
    q, cache, main, offs, tail = _case(lens, tails, H, G, d, torch.bfloat16, False, handle, 9)
    od = torch.tensor(offs, device="cuda")
    tl = torch.tensor(tails, dtype=torch.int32, device="cuda")
    args = fc.make_decode_args(q, *cache, od, 709, *tail, tl)
    need = fc._lib.fc_decode_workspace_bytes_ex(handle, ctypes.byref(args), None)
    assert need == fc.fc_decode_workspace_bytes(handle, args)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    fc.fc_decode_attention(handle, args, a, ws)
    assert fc._lib.fc_decode_attention_ex(handle, ctypes.byref(args), None, b.data_ptr(), ws.data_ptr(), ws.nbytes, fc._stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    want, tol = _definition(q, main, offs, tail, tails, 0, 0, torch.bfloat16, False)
    _check(_run(handle, q, cache, offs, tail, tails, 0, 0), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("four", [True, False])
def test_captured_step_follows_lengths_on_the_device(handle, four):
    lens, H, G, d = [300, 120], 2, 4, 64
    q, cache, main, offs, tail = _case(lens, [0, 0], H, G, d, torch.float16, four, handle, 21)
    od = torch.tensor(offs, device="cuda")
    tl = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    args, opt = fc.make_decode_args_ex(q, cache, od, 400, *tail, tl, window=64, sinks=2)
    ws = torch.empty(fc.fc_decode_workspace_bytes_ex(handle, args, opt), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fc.fc_decode_attention_ex(handle, args, opt, out, ws)
    for t in ([0, 0], [1, 80], [63, 64]):
        tl.copy_(torch.tensor(t, dtype=torch.int32))
        q.copy_(torch.randn(q.shape).half())
        graph.replay()
        torch.cuda.synchronize()
        want, tol = _definition(q, main, offs, tail, t, 64, 2, torch.float16, four)
        _check(out, want, tol)
    assert fc.fc_last_device_status(handle) == 0


# ---------------------------------------------------------------------------------------------- refusals, without a GPU
A = 1 << 20


def _args(**kw):
    a = fc.fc_decode_args(q=A, cache_k=A, cache_v=A, cache_rows=10, offsets=A, dtype=fc.FC_F16, batch=2, num_heads=2, num_q_heads=8,
                          head_dim=128, max_rows=10)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _opt(c4=None, window=0, sinks=0):
    o = fc.fc_decode_options(window=window, sinks=sinks)
    if c4 is not None:
        o.cache4 = ctypes.pointer(c4)
    return o


def test_decode_ex_refusals():
    h = ctypes.create_string_buffer(1 << 16)

    def call(a, o, out=A, ws=A, n=1 << 30):
        return fc._lib.fc_decode_attention_ex(h, ctypes.byref(a) if a is not None else None, ctypes.byref(o), out, ws, n, None)

    def size(a, o):
        return fc._lib.fc_decode_workspace_bytes_ex(h, ctypes.byref(a), ctypes.byref(o))

    def c4(**kw):
        c = fc.fc_cache4(A, A, A, A, 64, fc.FC_F16, 2, 128)
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    bad = [(dict(q=None), INVALID), (dict(offsets=None), INVALID), (dict(batch=0), INVALID), (dict(num_heads=0), INVALID),
           (dict(num_q_heads=0), INVALID), (dict(max_rows=-1), INVALID), (dict(q=A + 2), INVALID), (dict(dtype=fc.FC_F32), UNSUPPORTED),
           (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(num_q_heads=7), UNSUPPORTED),
           (dict(num_q_heads=34), UNSUPPORTED), (dict(batch=70000), UNSUPPORTED), (dict(max_rows=1 << 31), UNSUPPORTED),
           (dict(tail_k=A), INVALID), (dict(tail_k=A, tail_v=A, tail_len=A), INVALID),
           (dict(tail_k=A + 8, tail_v=A, tail_len=A, tail_capacity=4), INVALID)]
    for kw, want in bad:
        for o in (_opt(), _opt(c4(), 5, 1)):
            assert call(_args(**kw), o) == want and size(_args(**kw), o) == 0, kw
    for kw, want in ((dict(cache_k=None), INVALID), (dict(cache_v=A + 8), INVALID), (dict(cache_rows=0), INVALID),
                     (dict(cache_rows=1 << 31), UNSUPPORTED)):
        assert call(_args(**kw), _opt()) == want
        assert size(_args(**kw), _opt(c4())) > 0            # not read beside a 4-bit cache
    for kw, want in ((dict(dtype=fc.FC_BF16), INVALID), (dict(num_heads=4), INVALID), (dict(head_dim=64), INVALID),
                     (dict(codes_k=None), INVALID), (dict(capacity_rows=63), INVALID), (dict(head_dim=256), UNSUPPORTED)):
        assert call(_args(), _opt(c4(**kw))) == want, kw
    assert call(_args(), _opt(window=-1)) == INVALID and call(_args(), _opt(window=4, sinks=-1)) == INVALID
    assert call(None, _opt()) == INVALID
    for o in (_opt(), _opt(c4())):
        assert call(_args(), o, out=None) == INVALID and call(_args(), o, out=A + 8) == INVALID
        assert call(_args(), o, ws=None) == WORKSPACE and call(_args(), o, ws=A + 16) == WORKSPACE
        assert call(_args(), o, n=size(_args(), o) - 1) == WORKSPACE
    assert fc._lib.fc_decode_attention_ex(None, ctypes.byref(_args()), ctypes.byref(_opt()), A, A, 1 << 30, None) == INVALID


def test_rows_and_tails_past_the_last_int_are_refused():
    """Kept rows and tail of a sequence are counted together."""
    h, most = ctypes.create_string_buffer(1 << 16), 0x7fffffff - 4096

    def size(rows, cap, four):
        a = _args(cache_rows=10 if four else rows, tail_k=A, tail_v=A, tail_len=A, tail_capacity=cap)
        return fc._lib.fc_decode_workspace_bytes_ex(h, ctypes.byref(a), ctypes.byref(_opt(fc.fc_cache4(A, A, A, A, rows, fc.FC_F16, 2, 128) if four else None)))

    for four in (True, False):
        rows = most // 16 * 16 - 160
        assert size(rows, most - rows, four) > 0
        for cap in (most - rows + 1, 1 << 20, most, 0x7fffffff):
            assert size(rows, cap, four) == 0
            a = _args(cache_rows=rows, tail_k=A, tail_v=A, tail_len=A, tail_capacity=cap)
            o = _opt(fc.fc_cache4(A, A, A, A, rows, fc.FC_F16, 2, 128) if four else None)
            assert fc._lib.fc_decode_attention_ex(h, ctypes.byref(a), ctypes.byref(o), A, A, 1 << 30, None) == UNSUPPORTED
