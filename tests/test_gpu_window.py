"""fc_window_attention against its definition in 64 bits.

Tolerance, derived element by element.  A weight is rounded once to the type (eps / 2).  Scores are sums of d products in fp32,
each of the at most d + 8 additions off by 2^-23 (the tensor cores cut off) of the sum of the products' sizes, which moves every
weight by as much; twice, since the sum of the weights moves too.  Exponentials, sums of weights and the rest: 2^-16.  All of it
times the mean of the values' sizes under the weights; then half a step of the output's type."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2511_16786_b200 import binding as fc

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def _definition(q, k, v, nq, nk, window, sinks):
    """-> (out, tolerance) [Tq, Hq, d] in 64 bits; values that a query does not see do not touch it."""
    dtype = q.dtype
    eps = torch.finfo(dtype).eps
    q, k, v = (x.double().cuda() for x in (q, k, v))
    Hq, d = q.shape[1:]
    G = Hq // k.shape[1]
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    q0 = k0 = 0
    for n, m in zip(nq, nk):
        p = torch.arange(m - n, m, device="cuda")[:, None]
        j = torch.arange(m, device="cuda")[None]
        seen = (j <= p) & ((j > p - window) | (j < sinks))
        some = seen.any(1)
        for h in range(Hq if m else 0):
            qq, kk, vv = q[q0:q0 + n, h], k[k0:k0 + m, h // G], v[k0:k0 + m, h // G]
            s = (qq @ kk.t() / math.sqrt(d)).masked_fill(~seen, -math.inf)
            size = (qq.abs() @ kk.abs().t() / math.sqrt(d)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
            w = torch.exp(s - s.amax(1, keepdim=True))
            w = torch.where(some[:, None], w / w.sum(1, keepdim=True), 0.0)
            o, a = w @ vv, w @ vv.abs()
            out[q0:q0 + n, h] = o
            tol[q0:q0 + n, h] = a * (eps / 2 + 2 * (d + 8) * 2.0 ** -23 * size + 2.0 ** -16) + eps / 2 * o.abs() + torch.finfo(dtype).smallest_normal
        q0, k0 = q0 + n, k0 + m
    return out, tol


@pytest.fixture(scope="module")
def handle():
    h = fc.fc_create(0, 1024)
    yield h
    assert fc.fc_last_device_status(h) == 0
    fc.fc_destroy(h)


def _cu(n):
    return [int(x) for x in np.cumsum([0] + list(n))]


def _inputs(nq, nk, Hq, H, d, dtype, seed, peaked=1.0):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((sum(nq), Hq, d), generator=g) * peaked).to(dtype).cuda()
    k = (torch.randn((sum(nk), H, d), generator=g) + torch.randn((1, H, d), generator=g)).to(dtype).cuda()
    v = (torch.randn((sum(nk), H, d), generator=g) + 0.25).to(dtype).cuda()
    return q, k, v


def _run(handle, q, k, v, nq, nk, window, sinks, spare=3):
    args = fc.make_window_args(q, k, v, _cu(nq), _cu(nk), window, sinks)
    ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
    out = torch.full((q.shape[0] + spare, *q.shape[1:]), 123.0, dtype=q.dtype, device="cuda")
    fc.fc_window_attention(handle, args, out, ws)
    assert fc.fc_last_device_status(handle) == 0
    assert (out[q.shape[0]:] == 123).all()                      # rows behind the last query stay
    return out[:q.shape[0]]


def _check(out, want, tol):
    err = (out.double() - want).abs()
    assert torch.isfinite(out).all() and bool((err <= tol).all()), "worst error / tolerance %.3f" % float((err / tol.clamp(min=1e-300)).max())


SHAPES = [([1], [1], 1, 1, 1, 0), ([1, 5], [130, 5], 4, 4, 64, 4), ([128], [128], 2, 1, 1000, 0), ([129, 127], [129, 127], 7, 1, 64, 0),
          ([300], [300], 14, 2, 128, 4), ([517, 64, 1, 333], [517, 1000, 700, 2000], 8, 2, 100, 5), ([0, 70, 0], [10, 70, 0], 3, 1, 33, 2),
          ([40], [17], 2, 2, 8, 3), ([200, 9], [60, 0], 16, 1, 300, 0), ([700], [700], 3, 3, 1, 0), ([260], [900], 64, 1, 200, 130),
          ([513], [1500], 12, 1, 129, 300), ([2049], [2049], 4, 1, 5000, 0), ([16], [6000], 7, 1, 100000, 0), ([3, 90], [4000, 5], 8, 8, 700, 260),
          ([2, 1, 30] * 25, [2, 50, 31] * 25, 4, 2, 20, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk,Hq,H,window,sinks", SHAPES)
def test_window_matches_the_definition(handle, nq, nk, Hq, H, window, sinks, d, dtype):
    q, k, v = _inputs(nq, nk, Hq, H, d, dtype, sum(nq) + sum(nk) + d)
    _check(_run(handle, q, k, v, nq, nk, window, sinks), *_definition(q, k, v, nq, nk, window, sinks))


@pytest.mark.gpu
@pytest.mark.parametrize("peaked", [0.0, 8.0, 60.0])
def test_flat_and_peaked_scores(handle, peaked):
    nq, nk = [700], [900]
    q, k, v = _inputs(nq, nk, 4, 2, 128, torch.bfloat16, 5, peaked)
    _check(_run(handle, q, k, v, nq, nk, 300, 4), *_definition(q, k, v, nq, nk, 300, 4))


@pytest.mark.gpu
def test_scores_that_grow_along_the_keys_move_the_reference(handle):
    # every key tile has a larger maximum than the ones before it, by more than the slack, and then a smaller one
    n, d = 1200, 64
    q, k, v = _inputs([n], [n], 2, 1, d, torch.float16, 6)
    ramp = torch.arange(n, device="cuda").float()
    k = (k.float() * 0.1 + torch.where(ramp < 900, ramp / 60, 15 - (ramp - 900) / 30)[:, None, None]).half()
    q = (q.float() * 0.1 + 1.0).half()
    _check(_run(handle, q, k, v, [n], [n], n, 0), *_definition(q, k, v, [n], [n], n, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,G,window,sinks", [(128, 2, 100, 3), (64, 7, 1000, 0), (128, 1, 130, 140)])
def test_what_is_not_finite_reaches_who_sees_it_and_no_one_else(handle, d, G, window, sinks, dtype):
    nq, nk = [400, 90], [500, 90]
    H = 2
    q, k, v = _inputs(nq, nk, H * G, H, d, dtype, 9)
    want, tol = _definition(q, k, v, nq, nk, window, sinks)
    nan, inf = float("nan"), float("inf")
    v2, k2 = v.clone(), k.clone()
    # (sequence, key, head, channel or None for a key, what); sequence 1 lies behind sequence 0 in the same key tile
    marks = [(0, 1, 0, 5, nan), (0, 260, 0, d - 1, inf), (0, 261, 1, 0, -inf), (0, 499, 1, 7, nan), (1, 0, 0, 3, nan), (1, 89, 1, 33, inf),
             (0, 300, 1, None, nan)]
    hit = torch.zeros_like(want, dtype=torch.bool)
    for b, j, h, c, what in marks:
        at = _cu(nk)[b] + j
        if c is None:
            k2[at, h, 4] = what
        else:
            v2[at, h, c] = what
        p = torch.arange(nk[b] - nq[b], nk[b], device="cuda")
        sees = (j <= p) & ((j > p - window) | (j < sinks))
        rows = _cu(nq)[b] + torch.nonzero(sees).flatten()
        chans = slice(None) if c is None else slice(c, c + 1)
        hit[rows, h * G:(h + 1) * G, chans] = True
    out = _run(handle, q, k2, v2, nq, nk, window, sinks)
    bad = ~torch.isfinite(out)
    assert not (bad & ~hit).any(), "reached a query that does not see it"
    assert not (hit & ~bad).any(), "did not reach a query that sees it"
    err = (out.double() - want).abs()
    assert bool((err <= tol)[~hit].all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at,much", [((130,), 60.0), ((200,), 60.0), ((263, 391), 40.0), ((130, 131, 250, 255, 400), 25.0), ((640, 700), 300.0),
                                     ((134,), math.nan), ((201,), math.nan), ((255,), math.nan), ((128,), -math.inf)])
def test_single_keys_far_above_the_rest(handle, at, much, d, dtype):
    """In either half of a tile that all queries see whole: the reference moves in the middle of a tile, and NaN is seen
    wherever it stands.  `much`: how many powers of two such a key's weight is above the others'; every second head turns away."""
    nq, nk, g = 70, 900, torch.Generator().manual_seed(int(sum(at)))
    base = torch.randn(d, generator=g)
    q = base + 0.1 * torch.randn((nq, 2, d), generator=g)
    q[:, 1] *= -1
    k, v = (0.3 * torch.randn((nk, 1, d), generator=g) for _ in range(2))
    for i, key in enumerate(at):
        k[key] = base / (base @ base) * much * (1 + i / 4) * math.sqrt(d) * math.log(2.0) if math.isfinite(much) else much
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    out, (want, tol) = _run(handle, q, k, v, [nq], [nk], 5000, 0), _definition(q, k, v, [nq], [nk], 5000, 0)
    if math.isfinite(much):
        _check(out, want, tol)
    else:
        assert want.isnan().all() and out.isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("times", [1, 2])
def test_keys_whose_weight_passes_what_an_exponent_holds(handle, times, d, dtype):
    """Keys so far above the rest that 2^(score - reference) has no number of 32 bits, in the second tile of a block, which all
    queries see whole.  Each key-value head has other keys and another distance; with times = 2 there are blocks enough not
    to split the keys.  Every second query head turns away from the key."""
    places = [(128 + x,) for x in (6, 7, 62, 63, 70, 71, 126, 127)] + [(134, 135), (134, 190), (198, 255), (135, 199)]
    heads = [(at, much) for at in places for much in (130.0, 200.0, 270.0, 400.0, 512.0)]
    nq, nk, H, g = 70, 900, len(heads), torch.Generator().manual_seed(d)
    base = torch.randn((H, 1, d), generator=g)
    q = base * torch.tensor([1.0, -1.0])[:, None] + 0.1 * torch.randn((nq, H, 2, d), generator=g)
    k, v = (0.3 * torch.randn((nk, H, d), generator=g) for _ in range(2))
    for h, (at, much) in enumerate(heads):
        for i, key in enumerate(at):
            k[key, h] = base[h, 0] / (base[h, 0] @ base[h, 0]) * much * (1 + i / 4) * math.sqrt(d) * math.log(2.0)
    q, k, v = (x.to(dtype).cuda() for x in (q.reshape(nq, 2 * H, d).repeat(1, times, 1), k.repeat(1, times, 1), v.repeat(1, times, 1)))
    _check(_run(handle, q, k, v, [nq], [nk], 5000, 0), *_definition(q, k, v, [nq], [nk], 5000, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,nk", [(1, 20000), (80, 4000)])
@pytest.mark.parametrize("key", [0, 1])
@pytest.mark.parametrize("far", [16.0, 25.5, 28.0])
def test_many_keys_far_below_one_are_not_lost_in_half_numbers(handle, far, key, H, nk, d):
    """Thousands of keys whose weights are 2^-far of a first (or last) key's, which has a value of zero: the output is theirs.  A
    weight is a half number in units of 2^-7 of a row's largest at most, so the rounding is off by half a step of the small ones,
    2^-25 of those units: 2^-32 of the largest weight for every key, beside what holds for larger ones."""
    nq, g = 40, torch.Generator().manual_seed(int(far) + d)
    base = torch.randn(d, generator=g)
    q = (base + 0.02 * torch.randn((nq, H, d), generator=g)).half().cuda()
    k, v = 0.02 * torch.randn((nk, H, d), generator=g), 8 + 0.5 * torch.randn((nk, H, d), generator=g)
    at = 0 if key == 0 else nk - nq
    k[at] += base / (base @ base) * far * math.sqrt(d) * math.log(2.0)
    v[at] = 0.0
    k, v = k.half().cuda(), v.half().cuda()
    want, tol = _definition(q, k, v, [nq], [nk], nk, 0)
    tol += 2.0 ** -32 * v.double().abs().sum(0)                 # the largest weight is at most 1 of their sum
    _check(_run(handle, q, k, v, [nq], [nk], nk, 0), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("nq,nk", [([700], [700]), ([4], [6000])])
def test_scores_that_are_all_minus_infinity_are_undefined(handle, nq, nk, dtype):
    """0 / 0 by the definition, for the queries whose window holds such keys only; the others give them no weight."""
    d, window, g = 128, 300, torch.Generator().manual_seed(9)
    q = (torch.rand((nq[0], 2, d), generator=g) + 0.5).to(dtype).cuda()
    k, v = (torch.randn((nk[0], 1, d), generator=g).to(dtype).cuda() for _ in range(2))
    lo, hi = nk[0] - 650, nk[0] - 2
    k[lo:hi] = float("-inf")
    args = fc.make_window_args(q, k, v, [0] + nq, [0] + nk, window, 0)
    ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    fc.fc_window_attention(handle, args, out, ws)
    at = torch.arange(nq[0]) + nk[0] - nq[0]
    want = (at < hi) & (at - window + 1 >= lo)
    assert torch.equal(out.isnan().cpu(), want[:, None, None].expand(nq[0], 2, d))
    assert want.any() and not want.all()


@pytest.mark.gpu
def test_strided_views_and_rows_past_the_last_key(handle):
    # q, k, v out of one projection; keys behind the last sequence hold NaN
    T, Hq, H, d = 333, 4, 2, 64
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn((T + 40, (Hq + 2 * H) * d), generator=g).to(torch.bfloat16).cuda()
    q = qkv[:T, :Hq * d].view(T, Hq, d)
    k = qkv[:, Hq * d:(Hq + H) * d].view(T + 40, H, d)
    v = qkv[:, (Hq + H) * d:].view(T + 40, H, d)
    want, tol = _definition(q, k[:T], v[:T], [T], [T], 90, 2)
    qkv[T:] = float("nan")
    args = fc.make_window_args(q, k, v, [0, T], [0, T], 90, 2)
    ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
    out = torch.empty((T, Hq, d), dtype=q.dtype, device="cuda")
    fc.fc_window_attention(handle, args, out, ws)
    _check(out, want, tol)


@pytest.mark.gpu
def test_split_keys_give_the_same_as_one_block(handle):
    # few queries against many keys are split over blocks; the same queries among many others are not
    Hq, H, d, m = 4, 2, 128, 9000
    q, k, v = _inputs([20], [m], Hq, H, d, torch.bfloat16, 14)
    args = fc.make_window_args(q, k, v, [0, 20], [0, m], m, 0)
    assert fc.fc_window_workspace_bytes(handle, args) > 4096
    _check(_run(handle, q, k, v, [20], [m], m, 0), *_definition(q, k, v, [20], [m], m, 0))
    _check(_run(handle, q, k, v, [20], [m], 6000, 200), *_definition(q, k, v, [20], [m], 6000, 200))


@pytest.mark.gpu
def test_captured_on_another_stream_and_replayed(handle):
    nq, nk = [150, 20], [150, 4000]
    q, k, v = _inputs(nq, nk, 8, 2, 128, torch.float16, 3)
    args = fc.make_window_args(q, k, v, _cu(nq), _cu(nk), 2000, 4)
    ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fc.fc_window_attention(handle, args, out, ws)
    for scale in (1.0, -0.5):
        q.mul_(scale)
        v.add_(scale)
        graph.replay()
        torch.cuda.synchronize()
        _check(out, *_definition(q, k, v, nq, nk, 2000, 4))
    assert fc.fc_last_device_status(handle) == 0


@pytest.mark.gpu
def test_the_same_call_gives_the_same_bits(handle):
    nq, nk = [600, 33], [600, 5000]
    q, k, v = _inputs(nq, nk, 8, 2, 128, torch.bfloat16, 8)
    a, b = (_run(handle, q, k, v, nq, nk, 400, 4) for _ in range(2))
    assert torch.equal(a, b)


@pytest.mark.gpu
def test_calls_of_either_head_size_in_a_row(handle):
    """Each may begin while the one in front still runs, next to its blocks: the same bits as one by one."""
    calls = []
    for d, dtype, nq, nk, Hq, H in ((64, torch.float16, 300, 900, 4, 2), (128, torch.bfloat16, 200, 3000, 8, 2), (64, torch.bfloat16, 5, 4000, 2, 1),
                                    (128, torch.float16, 70, 70, 2, 2)):
        q, k, v = _inputs([nq], [nk], Hq, H, d, dtype, nk + d)
        args = fc.make_window_args(q, k, v, [0, nq], [0, nk], 500, 4)
        ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
        want = torch.empty_like(q)
        fc.fc_window_attention(handle, args, want, ws)
        torch.cuda.synchronize()
        calls.append((args, ws, want, (q, k, v)))
    outs = []
    for i in range(60):
        args, ws, want, _ = calls[(i * i + i // 7) % 4]
        outs.append((torch.empty_like(want), want))
        fc.fc_window_attention(handle, args, outs[-1][0], ws)
    assert all(torch.equal(a, b) for a, b in outs) and fc.fc_last_device_status(handle) == 0


# ---------------------------------------------------------------------------------------------- refusals, without a GPU
A = 1 << 20


def test_window_refusals():
    h = ctypes.create_string_buffer(1 << 16)
    cq, ck = (ctypes.c_int32 * 3)(0, 3, 9), (ctypes.c_int32 * 3)(0, 5, 9)

    def args(view=(), **kw):
        v = fc.fc_kv_view(A, A, 256, 128, fc.FC_F16, 2, 128, 2, ctypes.cast(ck, ctypes.POINTER(ctypes.c_int32)))
        for n, x in dict(view).items():
            setattr(v, n, x)
        a = fc.fc_window_args(q=A, q_stride_token=1024, q_stride_head=128, num_q_heads=8, window=4, sinks=1,
                              cu_seqlens_q=ctypes.cast(cq, ctypes.POINTER(ctypes.c_int32)), kv=ctypes.pointer(v))
        for n, x in kw.items():
            setattr(a, n, x)
        a._kept = v
        return a

    def call(a, out=A, ws=A, n=1 << 30):
        return fc._lib.fc_window_attention(h, ctypes.byref(a), out, ws, n, None)

    def size(a):
        return fc._lib.fc_window_workspace_bytes(h, ctypes.byref(a))

    assert size(args()) > 0
    for kw, want in ((dict(q=None), INVALID), (dict(kv=None), INVALID), (dict(cu_seqlens_q=None), INVALID), (dict(q=A + 8), INVALID),
                     (dict(window=0), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(num_q_heads=0), INVALID),
                     (dict(q_stride_token=100), INVALID), (dict(q_stride_head=0), INVALID), (dict(q_stride_token=-1024), INVALID),
                     (dict(num_q_heads=7), UNSUPPORTED), (dict(num_q_heads=130), UNSUPPORTED)):
        assert call(args(**kw)) == want and size(args(**kw)) == 0, kw
    for kw, want in ((dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 2), INVALID), (dict(cu_seqlens=None), INVALID),
                     (dict(batch=0), INVALID), (dict(num_heads=0), INVALID), (dict(stride_token=4), INVALID), (dict(stride_head=1 << 40), INVALID),
                     (dict(dtype=fc.FC_F32), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED)):
        assert call(args(view=kw)) == want and size(args(view=kw)) == 0, kw
    for cu in (cq, ck):
        for bad in ((1, 3, 9), (0, 9, 3), (0, 3, (1 << 30) + 1)):
            good = list(cu)
            cu[:] = bad
            assert call(args()) == INVALID, bad
            cu[:] = good
    assert call(args(), out=None) == INVALID and call(args(), out=A + 8) == INVALID
    assert call(args(), ws=None) == WORKSPACE and call(args(), ws=A + 128) == WORKSPACE and call(args(), n=size(args()) - 1) == WORKSPACE
    assert fc._lib.fc_window_attention(None, ctypes.byref(args()), A, A, 1 << 30, None) == INVALID
    assert fc._lib.fc_window_attention(h, None, A, A, 1 << 30, None) == INVALID
    cq[:] = (0, 0, 0)                                           # no queries: nothing to do, nothing launched
    assert call(args()) == 0
