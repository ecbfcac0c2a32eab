"""A model's layers from the prompt to its next tokens, as the operators are used together: positions, windowed attention of
the prefill, compression, 4-bit rows, and decoding steps that turn, append and attend, captured once and replayed."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

L, HQ, H, D = 2, 8, 2, 128
LENS = [700, 333]
WINDOW, SINKS, RHO, CAP, STEPS = 256, 4, 0.3, 40, 5


@pytest.fixture(scope="module")
def fc():
    from paper_2511_16786_b200 import binding
    return binding


def _attention(q, k, v, seen):
    """q [Hq, d], k and v [n, H, d] in 64 bits -> [Hq, d]."""
    out = np.zeros_like(q)
    for j in range(HQ):
        s = k[seen, j // (HQ // H)] @ q[j] / math.sqrt(D)
        w = np.exp(s - s.max())
        out[j] = w / w.sum() @ v[seen, j // (HQ // H)]
    return out


def _near(got, want, size, roundings):
    """Off by at most `roundings` roundings to bfloat16 (2^-8 each) of the values' size: one for a turned channel; two for
    attention, the weights' (an average of values is off by no more than its weights are, relatively) and the output's."""
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= roundings * 2.0 ** -8 * size).all(), "error %.2e of size" % (err / size).max()


def test_prompt_to_tokens(fc):
    T, B = sum(LENS), len(LENS)
    cu = [0, LENS[0], T]
    g = torch.Generator().manual_seed(7)
    dev = "cuda"
    handle = fc.fc_create(0, 1024)
    comp = fc.Compressor(L, H, D, cu, torch.bfloat16, RHO, min_keep=8)
    freq, scale = fc.fc_rotary_frequencies(D, 1e6, "yarn", 2.0, 512)
    pos = torch.cat([torch.arange(n) for n in LENS]).cuda()
    # ---- the prefill of every layer
    K, V = [], []
    for l in range(L):
        qkv = torch.randn((T, (HQ + 2 * H) * D), generator=g).to(torch.bfloat16).cuda()
        q, k, v = qkv[:, :HQ * D].view(T, HQ, D), qkv[:, HQ * D:(HQ + H) * D].view(T, H, D), qkv[:, (HQ + H) * D:].view(T, H, D)
        fc.fc_rotary(handle, fc.make_rotary_args(pos, freq, q=q, out_q=q, k=k, out_k=k, scale=scale))
        args = fc.make_window_args(q, k, v, cu, cu, WINDOW, SINKS)
        ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device=dev)
        out = torch.empty((T, HQ, D), dtype=torch.bfloat16, device=dev)
        fc.fc_window_attention(handle, args, out, ws)
        qd, kd, vd = (x.double().cpu().numpy() for x in (q, k, v))
        for b, n in enumerate(LENS):
            for i in (0, 5, WINDOW + 3, n - 1):
                j = np.arange(n)
                seen = (j <= i) & ((j > i - WINDOW) | (j < SINKS))
                want = _attention(qd[cu[b] + i], kd[cu[b]:cu[b + 1]], vd[cu[b]:cu[b + 1]], seen)
                _near(out[cu[b] + i], want, np.abs(vd[cu[b]:cu[b] + i + 1]).max(), 2)
        K.append(k.contiguous())
        V.append(v.contiguous())
    # ---- compression, then 4 bits; the kept rows are what the compressor says
    comp.compress(K, V)
    caches = comp.quantize()
    comp.check_device_status()
    off = comp.offsets.cpu()
    kept = []
    for l in range(L):
        n = int(off[l, B])
        k4, v4 = (torch.empty((n, H, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
        fc.fc_dequantize_cache(handle, caches[l], k4, v4)
        for x, y in ((comp.out_k[l, :n], k4), (comp.out_v[l, :n], v4)):
            half = x.float().unflatten(-1, (2, D // 2))
            step = (half.amax(-1) - half.amin(-1)) / 15
            moved = (half - y.float().unflatten(-1, (2, D // 2))).abs()
            # half a step (rounded up by at most 2^-7), and the value's rounding
            assert bool((moved <= step[..., None] * 0.504 + 2.0 ** -8 * half.abs().amax(-1, keepdim=True)).all())
        kept.append((k4.double().cpu().numpy(), v4.double().cpu().numpy()))
    assert comp.quantize()[0] is caches[0]
    # ---- decoding steps: one graph for all layers and steps; lengths, positions and rows live on the device
    qkv = torch.empty((L, B, HQ + 2 * H, D), dtype=torch.bfloat16, device=dev)
    tk, tv = (torch.zeros((L, B, CAP, H, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
    used = torch.zeros(B, dtype=torch.int32, device=dev)
    at = torch.tensor(LENS, device=dev)
    rows = torch.arange(B, device=dev) * CAP
    qr = torch.empty((L, B, HQ, D), dtype=torch.bfloat16, device=dev)
    out = torch.empty((L, B, HQ, D), dtype=torch.bfloat16, device=dev)
    rot, dec = [], []
    for l in range(L):
        q, k, v = qkv[l, :, :HQ], qkv[l, :, HQ:HQ + H], qkv[l, :, HQ + H:]
        rot.append(fc.make_rotary_args(at, freq, q=q, out_q=qr[l], k=k, out_k=tk[l].view(-1, H, D), v=v, out_v=tv[l].view(-1, H, D),
                                       out_rows=rows, scale=scale))
        most = int((off[l, 1:] - off[l, :-1]).max()) + CAP
        dec.append(fc.make_decode_args_ex(qr[l], caches[l], comp.offsets[l], most, tk[l], tv[l], used))
    ws = torch.empty(max(fc.fc_decode_workspace_bytes_ex(handle, *d) for d in dec), dtype=torch.uint8, device=dev)

    def step():
        used.add_(1)
        for l in range(L):
            fc.fc_rotary(handle, rot[l])
            fc.fc_decode_attention_ex(handle, *dec[l], out[l], ws)
        rows.add_(1)
        at.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for n in range(1, STEPS + 1):
        qkv.copy_(torch.randn(qkv.shape, generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for l in range(L):
            for b in range(B):
                k = np.concatenate((kept[l][0][off[l, b]:off[l, b + 1]], tk[l, b, :n].double().cpu().numpy()))
                v = np.concatenate((kept[l][1][off[l, b]:off[l, b + 1]], tv[l, b, :n].double().cpu().numpy()))
                # the newest key is the step's, turned to its position; its value as it is
                p = (LENS[b] + n - 1) * np.asarray(freq)
                x = qkv[l, b, HQ:HQ + H].double().cpu().numpy()
                c, s = np.cos(p) * scale, np.sin(p) * scale
                turned = np.concatenate((x[:, :64] * c - x[:, 64:] * s, x[:, 64:] * c + x[:, :64] * s), -1)
                _near(tk[l, b, n - 1], turned, np.abs(turned).max(), 1)
                assert torch.equal(tv[l, b, n - 1], qkv[l, b, HQ + H:])
                want = _attention(qr[l, b].double().cpu().numpy(), k, v, np.ones(len(k), dtype=bool))
                _near(out[l, b], want, np.abs(v).max(), 2)
        assert not tk[:, :, n:].any()
    assert fc.fc_last_device_status(handle) == 0
    comp.close()
    fc.fc_destroy(handle)


def test_outputs_that_do_not_fit_are_refused(fc):
    """By the binding, before anything is launched."""
    handle = fc.fc_create(0, 1024)
    q, k = torch.zeros((6, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros((6, 2, 64), dtype=torch.float16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    offs = torch.arange(7, device="cuda")
    window = fc.make_window_args(q, k, k, [0, 6], [0, 6], 4)
    decode = fc.make_decode_args_ex(q, (k, k), offs, 1)
    for out, room in ((torch.empty_like(q[:5]), ws), (torch.empty_like(q[:, :3]), ws), (torch.empty_like(q).float(), ws),
                      (torch.empty((6, 8, 64), dtype=q.dtype, device="cuda")[:, ::2], ws), (torch.empty_like(q, device="cpu"), ws),
                      (torch.empty_like(q), ws.cpu())):
        with pytest.raises(ValueError):
            fc.fc_window_attention(handle, window, out, room)
        with pytest.raises(ValueError):
            fc.fc_decode_attention_ex(handle, *decode, out, room)
    comp = fc.Compressor(1, 2, 64, [0, 6], torch.float16, 0.5)
    with pytest.raises(ValueError):
        comp.quantize()
    comp.close()
    fc.fc_destroy(handle)


def test_offsets_past_32_bits(fc):
    """Rows far into a cache of 4.6 GB, and tokens far apart in one of 5 GB."""
    handle = fc.fc_create(0, 1024)
    g = torch.Generator().manual_seed(3)
    n, Hn, d, cap = 300, 32, 128, 2_250_000
    k, v = (torch.randn((n, Hn, d), generator=g).to(torch.float16).cuda() for _ in range(2))
    q = torch.randn((1, Hn, d), generator=g).to(torch.float16).cuda()
    outs = []
    for rows, first in ((n, 0), (cap, cap - n)):
        cache = fc.Cache4.empty(rows, Hn, d, torch.float16)
        to = torch.arange(first, first + n, device="cuda")
        fc.fc_quantize_cache(handle, k, v, cache, out_rows=to)
        dec = fc.make_decode_args_ex(q, cache, torch.tensor([first, first + n], device="cuda"), n)
        ws = torch.empty(fc.fc_decode_workspace_bytes_ex(handle, *dec), dtype=torch.uint8, device="cuda")
        outs.append(torch.empty_like(q))
        fc.fc_decode_attention_ex(handle, *dec, outs[-1], ws)
        assert fc.fc_last_device_status(handle) == 0
        del cache
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].any())
    far = torch.empty(n * 2 ** 23, dtype=torch.float16, device="cuda")
    kv = [far.as_strided((n, Hn, d), (2 ** 23, d, 1), i * Hn * d) for i in range(3)]           # keys, values, queries
    for x, y in zip(kv, (k, v, k + v)):
        x.copy_(y)
    freq, _ = fc.fc_rotary_frequencies(d)
    pos = torch.arange(n, device="cuda")
    outs = []
    for kk, vv, qq in (kv, (k.clone(), v, k + v)):
        fc.fc_rotary(handle, fc.make_rotary_args(pos, freq, q=qq, out_q=qq, k=kk, out_k=kk))
        args = fc.make_window_args(qq, kk, vv, [0, n], [0, n], 90, 2)
        ws = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
        outs.append(torch.empty((n, Hn, d), dtype=torch.float16, device="cuda"))
        fc.fc_window_attention(handle, args, outs[-1], ws)
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].isfinite().all())
    assert fc.fc_last_device_status(handle) == 0
    fc.fc_destroy(handle)


def test_two_handles_on_two_streams_at_once(fc):
    import threading

    d, Hn, n = 128, 4, 900
    g = torch.Generator().manual_seed(12)
    data = [[torch.randn((n, heads, d), generator=g).to(torch.bfloat16).cuda() for heads in (8, Hn, Hn)] for _ in range(2)]
    torch.cuda.synchronize()

    def chain(q, k, v, times):
        handle = fc.fc_create(0, 1024)
        cache = fc.Cache4.empty(n, Hn, d, torch.bfloat16)
        args = fc.make_window_args(q, k, v, [0, n], [0, n], 200, 4)
        offs = torch.tensor([0, 500, 500, n], device="cuda")
        dec = fc.make_decode_args_ex(q[:3].contiguous(), cache, offs, n)
        wa = torch.empty(fc.fc_window_workspace_bytes(handle, args), dtype=torch.uint8, device="cuda")
        wd = torch.empty(fc.fc_decode_workspace_bytes_ex(handle, *dec), dtype=torch.uint8, device="cuda")
        seen = []
        for _ in range(times):
            a, b = torch.empty_like(q), torch.empty_like(q[:3])
            fc.fc_window_attention(handle, args, a, wa)
            fc.fc_quantize_cache(handle, k, v, cache)
            fc.fc_decode_attention_ex(handle, *dec, b, wd)
            seen.append((a, b))
        assert fc.fc_last_device_status(handle) == 0
        fc.fc_destroy(handle)
        return seen

    want = [chain(*x, 1)[0] for x in data]
    got = [None, None]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = chain(*data[i], 30)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        for a, b in got[i]:
            assert torch.equal(a, want[i][0]) and torch.equal(b, want[i][1])


def test_nothing_to_do(fc):
    """Empty tensors, which have no address, in every place that may be empty."""
    handle = fc.fc_create(0, 1024)
    empty = torch.empty((0, 4, 64), dtype=torch.float16, device="cuda")
    some = torch.ones((5, 4, 64), dtype=torch.float16, device="cuda")
    freq, _ = fc.fc_rotary_frequencies(64)
    fc.fc_rotary(handle, fc.make_rotary_args(torch.empty(0, dtype=torch.int64, device="cuda"), freq, q=empty, out_q=empty, k=empty, out_k=empty))
    cache = fc.Cache4.empty(16, 4, 64, torch.float16)
    fc.fc_quantize_cache(handle, empty, empty, cache)
    fc.fc_dequantize_cache(handle, cache, empty, empty)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for q, k, cq, ck in ((empty, empty, [0, 0], [0, 0]), (empty, some, [0, 0], [0, 5]), (some, empty, [0, 2, 5], [0, 0, 0])):
        args = fc.make_window_args(q, k, k, cq, ck, 3)
        assert 0 < fc.fc_window_workspace_bytes(handle, args) <= ws.nbytes
        out = torch.full_like(q, 7.0)
        fc.fc_window_attention(handle, args, out, ws)
        assert not out.any()                                       # queries that see nothing
    offs = torch.zeros(6, dtype=torch.int64, device="cuda")
    for held in (cache, (some, some)):
        out = torch.full_like(some, 7.0)
        dec = fc.make_decode_args_ex(some, held, offs, 0)
        fc.fc_decode_attention_ex(handle, *dec, out, torch.empty(fc.fc_decode_workspace_bytes_ex(handle, *dec), dtype=torch.uint8, device="cuda"))
        assert not out.any()
    assert fc.fc_last_device_status(handle) == 0
    fc.fc_destroy(handle)
