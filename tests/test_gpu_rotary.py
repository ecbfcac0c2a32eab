"""fc_rotary against its definition in 64 bits.

Tolerance, derived: a turned channel is a c - b s in fp32, rounded once to the type.  The remainder of the angle in turns
is rounded to fp32 (2^-26 turns, 9.4e-8 radians), sine and cosine carry one rounding of 2^-24, their product with the scale
one, each product and the sum one: at most 5e-7 * (|a| + |b|) * scale in all, then half a step of the type (eps/2 of the
value, or half the smallest step)."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


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


def _want(x, pos, freq, scale=1.0, interleaved=False, inverse=False, sections=None):
    """-> (value, |a| + |b| of every channel's pair) in 64 bits."""
    y = x.double().cpu().numpy().copy()
    r = 2 * len(freq)
    axis = np.repeat(np.arange(3), sections) if sections else np.zeros(len(freq), dtype=int)
    p = pos.cpu().numpy().reshape(-1, y.shape[0]).astype(np.float64)
    angle = p[axis].T * np.asarray(freq, dtype=np.float64)          # [T, pairs]
    c, s = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale * (-1 if inverse else 1)
    ia, ib = (np.arange(0, r, 2), np.arange(1, r, 2)) if interleaved else (np.arange(r // 2), np.arange(r // 2, r))
    a, b = y[..., ia].copy(), y[..., ib].copy()
    size = np.zeros_like(y)
    size[..., ia] = size[..., ib] = (np.abs(a) + np.abs(b)) * abs(scale)
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y, size


def _check(got, want, size, dtype):
    err = np.abs(got.double().cpu().numpy() - want)
    bound = 5e-7 * size + torch.finfo(dtype).eps / 2 * np.abs(want) * (1 + 1e-6) + TINY[dtype] / 2
    assert (err <= bound).all(), "worst excess %.3e" % (err - bound).max()


def _inputs(T, Hq, H, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((T, h, d), generator=g).to(dtype).cuda() for h in (Hq, H, H)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,Hq,H,d,r,inter,inverse,sections,first", [
    (1, 1, 1, 64, 64, False, False, None, 0),
    (1, 28, 4, 128, 128, False, False, (16, 24, 24), 77),
    (7, 3, 1, 128, 64, True, False, None, 123456),
    (33, 4, 2, 64, 24, False, True, None, 5000),         # the rotated part does not split into 16-byte pieces
    (5, 2, 2, 128, 18, True, False, (2, 3, 4), 10 ** 6),
    (2, 1, 1, 64, 2, False, False, None, 1 << 40),
    (601, 2, 1, 192, 160, True, False, None, 0),         # several tokens per block, the last block not full
    (1201, 1, 3, 256, 256, False, True, (0, 100, 28), 31)])
def test_rotary_matches_the_definition(fc, handle, T, Hq, H, d, r, inter, inverse, sections, first, dtype):
    q, k, _ = _inputs(T, Hq, H, d, dtype, T + d + r)
    freq, scale = fc.fc_rotary_frequencies(r, 1e4, "yarn", 4.0, 4096)
    g = torch.Generator().manual_seed(T)
    pos = (first + torch.randint(0, 5000, ((3, T) if sections else (T,)), generator=g)).cuda()
    oq, ok = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    args = fc.make_rotary_args(pos, freq, q=q, out_q=oq, k=k, out_k=ok, scale=scale, interleaved=inter, inverse=inverse, sections=sections)
    fc.fc_rotary(handle, args)
    assert fc.fc_last_device_status(handle) == 0
    for x, out in ((q, oq), (k, ok)):
        want, size = _want(x, pos, freq, scale, inter, inverse, sections)
        _check(out, want, size, dtype)
        assert torch.equal(out[..., r:], x[..., r:])


def test_rotary_in_place_on_strided_rows(fc, handle):
    # q, k and v of one projection, [T][(Hq + 2H) d]; turned where they are, v untouched, what lies beside untouched
    T, Hq, H, d = 37, 4, 2, 128
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((T, (Hq + 2 * H) * d + 16), generator=g).to(torch.bfloat16).cuda()
    before = qkv.clone()
    q = qkv[:, :Hq * d].view(T, Hq, d)
    k = qkv[:, Hq * d:(Hq + H) * d].view(T, H, d)
    pos = torch.arange(T, device="cuda")
    freq, _ = fc.fc_rotary_frequencies(d, 1e6)
    fc.fc_rotary(handle, fc.make_rotary_args(pos, freq, q=q, out_q=q, k=k, out_k=k))
    for now, was in ((q, before[:, :Hq * d].view(T, Hq, d)), (k, before[:, Hq * d:(Hq + H) * d].view(T, H, d))):
        want, size = _want(was, pos, freq)
        _check(now, want, size, torch.bfloat16)
    assert torch.equal(qkv[:, (Hq + H) * d:], before[:, (Hq + H) * d:])
    # and back: two roundings of the type, and the error of either pass
    fc.fc_rotary(handle, fc.make_rotary_args(pos, freq, q=q, out_q=q, inverse=True))
    was = before[:, :Hq * d].view(T, Hq, d).double().cpu().numpy()
    _, size = _want(before[:, :Hq * d].view(T, Hq, d), pos, freq)
    err = np.abs(q.double().cpu().numpy() - was)
    assert (err <= (2.0 ** -8 * 1.5 + 2e-6) * size + 2.0 ** -8 * np.abs(was)).all()


def test_rotary_appends_rows_and_leaves_the_others(fc, handle):
    B, cap, Hq, H, d = 6, 5, 4, 2, 64
    q, k, v = _inputs(B, Hq, H, d, torch.float16, 8)
    tail_k, tail_v = (torch.full((B, cap, H, d), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    used = torch.tensor([0, 4, 2, 1, 3, 0], device="cuda")
    rows = torch.arange(B, device="cuda") * cap + used
    rows[3] = -1                                         # padded
    pos = torch.tensor([9, 0, 100, 5, 31, 2], device="cuda")
    freq, _ = fc.fc_rotary_frequencies(d, 1e4)
    oq = torch.empty_like(q)
    args = fc.make_rotary_args(pos, freq, q=q, out_q=oq, k=k, out_k=tail_k.view(-1, H, d), v=v, out_v=tail_v.view(-1, H, d), out_rows=rows)
    fc.fc_rotary(handle, args)
    want, size = _want(k, pos, freq)
    for b in range(B):
        for c in range(cap):
            if b != 3 and c == int(used[b]):
                _check(tail_k[b, c], want[b], size[b], torch.float16)
                assert torch.equal(tail_v[b, c], v[b])
            else:
                assert (tail_k[b, c] == 7).all() and (tail_v[b, c] == 7).all()
    wq, sq = _want(q, pos, freq)
    _check(oq, wq, sq, torch.float16)
    assert fc.fc_last_device_status(handle) == 0
    # a row behind the tail is left out and said; the others are written
    rows[5] = B * cap
    fc.fc_rotary(handle, args)
    assert fc.fc_last_device_status(handle) == 6
    assert fc.fc_last_device_status(handle) == 0


def test_rotary_gradient(fc, handle):
    # y = R x is linear, so differences of the sum <w, y> give the gradient R^T w, which is the inverse call on w
    T, d = 3, 64
    x, w, _ = (t.double() for t in _inputs(T, 1, 1, d, torch.float32, 4))
    pos = torch.tensor([1, 50, 999], device="cuda")
    freq, scale = fc.fc_rotary_frequencies(d, 1e4, "yarn", 8.0, 2048)

    def turned(t, inverse=False):
        t = t.float().contiguous()
        out = torch.empty_like(t)
        fc.fc_rotary(handle, fc.make_rotary_args(pos, freq, q=t, out_q=out, scale=scale, inverse=inverse))
        return out.double()

    grad = turned(w, True)
    want, size = _want(w.float(), pos, freq, scale, inverse=True)
    _check(grad, want, size, torch.float32)
    for t, c in ((0, 0), (1, 31), (2, 63), (2, 32)):
        step = torch.zeros_like(x)
        step[t, 0, c] = 1.0
        diff = ((turned(x + step) - turned(x - step)) * w).sum() / 2
        # each of the two passes: 2^-23 of values below 8, times |w| over the pair
        assert abs(float(diff - grad[t, 0, c])) < 1e-5


def test_rotary_captured_and_on_another_stream(fc, handle):
    q, k, v = _inputs(16, 8, 2, 128, torch.bfloat16, 6)
    pos = torch.zeros(16, dtype=torch.int64, device="cuda")
    freq, _ = fc.fc_rotary_frequencies(128, 1e6)
    oq, ok, ov = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    args = fc.make_rotary_args(pos, freq, q=q, out_q=oq, k=k, out_k=ok, v=v, out_v=ov)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fc.fc_rotary(handle, args)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(oq, q) and torch.equal(ok, k) and torch.equal(ov, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fc.fc_rotary(handle, args)
    pos.add_(torch.arange(16, device="cuda"))            # the graph reads positions when it is replayed
    graph.replay()
    want, size = _want(q, pos, freq)
    _check(oq, want, size, torch.bfloat16)
    assert torch.equal(ov, v)


def test_rotary_argument_checks_of_the_binding(fc):
    q, k, v = _inputs(4, 2, 1, 64, torch.bfloat16, 1)
    pos = torch.arange(4, device="cuda")
    freq, _ = fc.fc_rotary_frequencies(64)
    for kw in (dict(), dict(q=q), dict(q=q, out_q=torch.empty_like(q)[:3]), dict(q=q, out_q=q.float()), dict(k=k, out_k=k, v=v),
               dict(k=k, out_k=k, v=q, out_v=q), dict(q=q, out_q=q, out_rows=pos), dict(k=k, out_k=k, out_rows=pos.int()),
               dict(q=q.transpose(0, 2), out_q=q.transpose(0, 2)), dict(q=q, out_q=q, sections=(10, 11, 11)),
               dict(q=q, out_q=q.cpu())):
        with pytest.raises(ValueError):
            fc.make_rotary_args(pos, freq, **kw)
    with pytest.raises(ValueError):
        fc.make_rotary_args(pos.int(), freq, q=q, out_q=q)
    with pytest.raises(ValueError):
        fc.make_rotary_args(pos[:3], freq, q=q, out_q=q)
