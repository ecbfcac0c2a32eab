"""The operators around the compressed cache, as a user of the library calls them, for timing and for comparing with their plain forms.

* ``rotary``    rotary positions of q and k: a whole prefill, or the rows of a decoding step, rotated and appended to the caches' tails.
* ``quantize``  rows of a compacted cache into 4 bits, and the values they stand for back into 16 bits.
* ``decode``    attention of one decoding step over rows held in 4 or in 16 bits and an uncompressed tail, with or without a window and sinks.
* ``window``    attention of a prefill (or of a chunk of it) with a sliding window and a few first tokens that stay visible.

A 4-bit row of d channels is two halves with a (scale, min) pair each, value = min + scale * code; `_nibble` has the order of the codes.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_BLOCK = 128                      # queries per block of the plain windowed attention


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _rotary(name, tokens, q_heads, heads, dtype, **more):
    case = dict(name=name, kind="rotary", tokens=tokens, q_heads=q_heads, heads=heads, dim=128, rotary=128, interleaved=False,
                scaling="none", base=1e6, factor=1.0, original=0, first=0, sections="", append=False, inverse=False, dtype=dtype)
    case.update(more)
    return case


def _decode(name, bits, rows, tails, heads, q_heads, dtype, **more):
    case = dict(name=name, kind="decode", bits=bits, rows=rows, tails=tails, heads=heads, q_heads=q_heads, dim=128, window=0, sinks=0,
                dtype=dtype)
    case.update(more)
    return case


def listed():
    return [
        # a decoding step of a batch of eight: q rotated, k rotated and appended with v; all launch and latency
        _rotary("rotary_step_8_bf16", 8, 28, 4, "bf16", append=True, first=30000),
        # the prefill of a long multi-image prompt: three position axes (time, height, width) over sections of the head
        _rotary("rotary_prefill_32768_bf16", 32768, 28, 4, "bf16", sections="16,24,24"),
        # keys far out taken back to position 0: half of the head, interleaved pairs, frequencies scaled for long contexts
        _rotary("rotary_partial_yarn_f16", 5001, 32, 32, "f16", rotary=64, interleaved=True, scaling="yarn", factor=4.0, original=32768,
                first=100000, inverse=True, base=1e4),
        # one layer of a compacted cache: a fifth of 32768 tokens
        dict(name="quantize_6554_bf16", kind="quantize", rows=6554, spare=57, heads=4, dim=128, dtype="bf16"),
        # a layer of a multi-head model's whole prompt
        dict(name="quantize_16384_f16_mha", kind="quantize", rows=16384, spare=0, heads=32, dim=128, dtype="f16"),
        # a step over a short kept cache: latency
        _decode("decode4_820_f16", 4, "820", "", 4, 28, "f16"),
        # a small batch on kept rows with the tokens generated since
        _decode("decode4_kept_tails_bf16", 4, "1638,205,3277,820", "17,64,1,100", 4, 28, "bf16"),
        # whole caches of a batch of videos of unlike lengths: only the bits are saved
        _decode("decode4_ragged_long_bf16", 4, "32092,26864,10164,8221,38158,13763,53602,6946", "", 4, 28, "bf16"),
        # as many KV heads as query heads: the most bytes per token
        _decode("decode4_mha_f16", 4, "16384,16384,9001,1", "5,0,130,64", 32, 32, "f16"),
        # a windowed layer's step: the first tokens and the last few thousand rows of uncompressed caches
        _decode("decode_window_bf16", 16, "65536,30001,777", "100,64,1", 4, 28, "bf16", window=4096, sinks=4),
        # a batch of ordinary requests, some of them chunks behind rows that are cached already
        dict(name="window_ragged_f16", kind="window", q_lens="517,1024,64,1999,333,1,100,2311", k_lens="517,1024,1000,1999,4096,700,100,2311",
             heads=4, q_heads=16, dim=64, window=512, sinks=4, dtype="f16"),
        # the prefill of a windowed layer over a long prompt
        dict(name="window_32768_bf16", kind="window", q_lens="32768", k_lens="32768", heads=4, q_heads=28, dim=128, window=4096, sinks=4,
             dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("rotary", "quantize", "decode", "window"), weights=(2, 1, 4, 3))[0]
    dtype = rng.choice(("f16", "bf16"))
    dim = rng.choice((64, 128, 128))
    heads = rng.choice((1, 2, 4, 8))
    q_heads = heads * rng.choice((1, 2, 3, 4, 7, 8, 12, 16))
    if kind == "rotary":
        scaling = rng.choice(("none", "linear", "ntk", "yarn", "bands"))
        factor = 1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0, 2.5))
        append = rng.random() < 0.3
        tokens = rng.randint(1, 64) if append else _log_int(rng, 1, 20000)
        rotary = rng.choice((dim, dim, dim // 2, dim // 4, 24, 18))
        sections = ""
        if rng.random() < 0.3:
            a = rng.randint(1, rotary // 2 - 2)
            b = rng.randint(1, rotary // 2 - a - 1)
            sections = "%d,%d,%d" % (a, b, rotary // 2 - a - b)
        return dict(kind="rotary", tokens=tokens, q_heads=min(q_heads, 32), heads=heads, dim=dim, rotary=rotary,
                    interleaved=rng.random() < 0.5, scaling=scaling, base=rng.choice((1e4, 5e5, 1e6)), factor=factor,
                    original=rng.choice((4096, 32768)), first=rng.choice((0, 0, rng.randint(1, 1000000))), sections=sections,
                    append=append, inverse=not append and rng.random() < 0.3, dtype=rng.choice(("f16", "bf16", "f32")))
    if kind == "quantize":
        return dict(kind="quantize", rows=_log_int(rng, 1, 60000 // heads * 4), spare=rng.randint(0, 99), heads=heads, dim=dim, dtype=dtype)
    if kind == "decode":
        batch = rng.choice((1, 1, 2, 4, 8))
        most = 400000 // (batch * heads)
        rows = [0 if batch > 1 and rng.random() < 0.1 else _log_int(rng, 1, most) for _ in range(batch)]
        tails = [rng.choice((0, rng.randint(1, 300))) for _ in range(batch)]
        window, sinks = rng.choice(((0, 0), (0, 0), (_log_int(rng, 1, 5000), rng.choice((0, 1, 4, 37, 200)))))
        return dict(kind="decode", bits=rng.choice((4, 4, 16)), rows=",".join(map(str, rows)),
                    tails=rng.choice(("", ",".join(map(str, tails)))), heads=heads, q_heads=q_heads, dim=dim, window=window, sinks=sinks,
                    dtype=dtype)
    batch = rng.choice((1, 1, 2, 5))
    q_lens = [_log_int(rng, 1, 8000 // batch) for _ in range(batch)]
    k_lens = [n + rng.choice((0, 0, _log_int(rng, 1, 4000))) for n in q_lens]
    if rng.random() < 0.1:
        k_lens[0] = max(1, q_lens[0] // 2)           # more queries than keys: the first ones see nothing
    return dict(kind="window", q_lens=",".join(map(str, q_lens)), k_lens=",".join(map(str, k_lens)), heads=heads,
                q_heads=min(q_heads, 32 if 32 % heads == 0 else heads), dim=dim, window=_log_int(rng, 1, 12000),
                sinks=rng.choice((0, 1, 4, 16, 130)), dtype=dtype)


# ------------------------------------------------------------------------------------------------ what a program has in hand
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _rows(g, n, heads, dim, dtype):
    """Keys and values: keys with a mean of their own per channel and a few wide channels, one row in a hundred far out."""
    wide = 1.0 + 4.0 * (torch.rand((heads, dim), generator=g, device="cuda") < 0.05)
    mean = torch.randn((heads, dim), generator=g, device="cuda")
    far = 1.0 + 2.0 * (torch.rand((n, 1, 1), generator=g, device="cuda") < 0.01)
    k = (torch.randn((n, heads, dim), generator=g, device="cuda") * wide * 0.5 + mean) * far
    v = torch.randn((n, heads, dim), generator=g, device="cuda") * far
    return k.to(dtype), v.to(dtype)


def _frequencies(case):
    """Radians per position of every pair and the factor on cosine and sine."""
    r, base, f, orig = case["rotary"], case["base"], case["factor"], case["original"]
    kind = case["scaling"]
    if kind == "ntk":
        base = base * f ** (r / (r - 2))
    plain = [base ** (-2.0 * j / r) for j in range(r // 2)]
    if kind == "linear":
        return [x / f for x in plain], 1.0
    if kind == "yarn":
        def at(turns):
            return r * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        hi = hi if hi > lo else lo + 0.001
        mix = [min(1.0, max(0.0, (j - lo) / (hi - lo))) for j in range(r // 2)]
        return [x * (1 - m) + x / f * m for x, m in zip(plain, mix)], 0.1 * math.log(f) + 1.0
    if kind == "bands":
        def scaled(x):
            share = min(1.0, max(0.0, (orig * x / (2 * math.pi) - 1.0) / (4.0 - 1.0)))
            return x * share + x / f * (1 - share)
        return [scaled(x) for x in plain], 1.0
    return plain, 1.0


def _nibble(dim, values):
    """Place of every channel's code in a row of dim / 2 bytes, counted in nibbles, low nibble first."""
    if values:                                        # value rows: eight runs, run g holds channels g, g + 8, g + 16, ...
        return [(c % 8) * (dim // 8) + c // 8 for c in range(dim)]
    # key rows: four runs, run t holds channels 4t .. 4t+3 of every 16; two such quads share a word of eight nibbles
    return [(c // 4 % 4) * (dim // 4) + (c // 32) * 8 + 4 * (c % 2) + c % 4 // 2 + 2 * (c // 16 % 2) for c in range(dim)]


def _quantized(x):
    """Codes, scales and minima of the rows' halves: the scale is (max - min) / 15 rounded up to the rows' type, codes go half to even."""
    half = x.unflatten(-1, (2, x.shape[-1] // 2))
    lo, hi = half.amin(-1), half.amax(-1)
    want = (hi.double() - lo.double()) / 15.0
    scale = want.to(x.dtype)
    scale = torch.where(scale.double() < want, (scale.view(torch.int16) + 1).view(x.dtype), scale)
    step = torch.where(scale == 0, torch.ones_like(scale), scale).double()
    codes = torch.round((half.double() - lo.double().unsqueeze(-1)) / step.unsqueeze(-1))
    return codes.to(torch.uint8).flatten(-2), scale, lo


def _packed(x, capacity, values):
    """A 4-bit cache of rows [n, heads, dim]: codes [heads, capacity, dim / 2], and [heads, capacity, 4] of (scale, min) pairs."""
    n, heads, dim = x.shape
    codes, scale, lo = _quantized(x)
    at = torch.empty(dim, dtype=torch.int64)
    at[torch.tensor(_nibble(dim, values))] = torch.arange(dim)
    nib = codes[..., at.cuda()].unflatten(-1, (dim // 2, 2))
    out = torch.zeros((heads, capacity, dim // 2), dtype=torch.uint8, device="cuda")
    out[:, :n] = (nib[..., 0] | (nib[..., 1] << 4)).transpose(0, 1)
    par = torch.zeros((heads, capacity, 4), dtype=x.dtype, device="cuda")
    par[:, :n] = torch.stack((scale, lo), -1).flatten(-2).transpose(0, 1)
    return out, par


def _capacity(rows):
    return (max(rows, 1) + 15) // 16 * 16


def _handle():
    global _kept
    from paper_2511_16786_b200 import binding as fc
    if _kept is None:
        _kept = fc.fc_create(torch.cuda.current_device(), 1024)
    return fc, _kept


_kept = None


def prepare(case, seed):
    g = _generator(seed)
    dtype, dim, heads = _DTYPES[case["dtype"]], case["dim"], case["heads"]
    s = dict(case=case)
    if case["kind"] == "rotary":
        n, hq = case["tokens"], case["q_heads"]
        s["q"], s["k"], s["v"] = (_normal(g, (n, h, dim), dtype) for h in (hq, heads, heads))
        axes = 3 if case["sections"] else 1
        step = torch.arange(n, device="cuda", dtype=torch.int64)
        if axes == 3:                                 # an image's patches: one time, rows of 64 patches
            s["positions"] = case["first"] + torch.stack((step // 4096, step // 64 % 64, step % 64))
        elif case["append"]:                          # every sequence of the batch is somewhere else
            s["positions"] = case["first"] + torch.randint(0, 5000, (1, n), generator=g, device="cuda")
        else:
            s["positions"] = case["first"] + step[None]
        s["freq"], s["scale"] = _frequencies(case)
        s["out_q"] = torch.empty_like(s["q"])
        if case["append"]:                            # [batch, capacity, heads, dim], seen as rows
            s["out_k"], s["out_v"] = (torch.zeros((n * 128, heads, dim), dtype=dtype, device="cuda") for _ in range(2))
            s["out_rows"] = 128 * step + torch.randint(0, 128, (n,), generator=g, device="cuda")
        else:
            s["out_k"] = torch.empty_like(s["k"])
    elif case["kind"] == "quantize":
        rows = case["rows"] + case["spare"]
        s["k"], s["v"] = _rows(g, rows, heads, dim, dtype)
        s["used"] = torch.tensor([case["rows"]], dtype=torch.int64, device="cuda")
        s["out_k"], s["out_v"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        cap = _capacity(rows)
        s["cache"] = [torch.zeros((heads, cap, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2)] + \
                     [torch.zeros((heads, cap, 4), dtype=dtype, device="cuda") for _ in range(2)]
    elif case["kind"] == "decode":
        rows, tails = _ints(case["rows"]), _ints(case["tails"])
        k, v = _rows(g, max(sum(rows), 1), heads, dim, dtype)
        s["q"] = _normal(g, (len(rows), case["q_heads"], dim), dtype)
        s["offsets"] = torch.tensor([sum(rows[:b]) for b in range(len(rows) + 1)], dtype=torch.int64, device="cuda")
        s["tail_k"] = s["tail_v"] = s["tail_len"] = None
        if tails:
            tk, tv = _rows(g, len(rows) * 320, heads, dim, dtype)
            s["tail_k"], s["tail_v"] = (t.view(len(rows), 320, heads, dim) for t in (tk, tv))
            s["tail_len"] = torch.tensor(tails, dtype=torch.int32, device="cuda")
        if case["bits"] == 4:
            cap = _capacity(k.shape[0])
            (ck, pk), (cv, pv) = _packed(k, cap, False), _packed(v, cap, True)
            s["cache"] = [ck, cv, pk, pv]
        else:
            s["cache"] = [k, v]
        s["out"] = torch.empty_like(s["q"])
    else:
        nq, nk = _ints(case["q_lens"]), _ints(case["k_lens"])
        s["q"] = _normal(g, (sum(nq), case["q_heads"], dim), dtype)
        s["k"], s["v"] = _rows(g, sum(nk), heads, dim, dtype)
        s["out"] = torch.empty_like(s["q"])
    if own:                                           # what such a program keeps: the handle, argument blocks, workspaces
        fc, h = _handle()
        s["handle"] = h
        if case["kind"] == "rotary":
            freq, scale = fc.fc_rotary_frequencies(case["rotary"], case["base"], case["scaling"], case["factor"], case["original"])
            s["args"] = fc.make_rotary_args(
                s["positions"], freq, q=s["q"], out_q=s["out_q"], k=s["k"], out_k=s["out_k"],
                v=s["v"] if case["append"] else None, out_v=s["out_v"] if case["append"] else None, out_rows=s.get("out_rows"),
                scale=scale, interleaved=case["interleaved"], inverse=case["inverse"], sections=_ints(case["sections"]) or None)
        elif case["kind"] == "quantize":
            s["cache4"] = fc.Cache4(*s["cache"])
        elif case["kind"] == "decode":
            most = max(r + t for r, t in zip(_ints(case["rows"]), _ints(case["tails"]) or [0] * len(_ints(case["rows"]))))
            cache = fc.Cache4(*s["cache"]) if case["bits"] == 4 else tuple(s["cache"])
            s["args"], s["options"] = fc.make_decode_args_ex(s["q"], cache, s["offsets"], most, s["tail_k"], s["tail_v"], s["tail_len"],
                                                             window=case["window"], sinks=case["sinks"])
            need = fc.fc_decode_workspace_bytes_ex(h, s["args"], s["options"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        else:
            cu = [[sum(n[:b]) for b in range(len(n) + 1)] for n in (_ints(case["q_lens"]), _ints(case["k_lens"]))]
            s["args"] = fc.make_window_args(s["q"], s["k"], s["v"], cu[0], cu[1], case["window"], case["sinks"])
            s["workspace"] = torch.empty(fc.fc_window_workspace_bytes(h, s["args"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if not own:
        return _PLAIN[case["kind"]](s, case)
    from paper_2511_16786_b200 import binding as fc
    if case["kind"] == "rotary":
        fc.fc_rotary(s["handle"], s["args"])
        return [s["out_q"], s["out_k"], s["out_v"]] if case["append"] else [s["out_q"], s["out_k"]]
    if case["kind"] == "quantize":
        fc.fc_quantize_cache(s["handle"], s["k"], s["v"], s["cache4"], used=s["used"])
        fc.fc_dequantize_cache(s["handle"], s["cache4"], s["out_k"], s["out_v"], used=s["used"])
        return [s["out_k"], s["out_v"]]
    if case["kind"] == "decode":
        fc.fc_decode_attention_ex(s["handle"], s["args"], s["options"], s["out"], s["workspace"])
    else:
        fc.fc_window_attention(s["handle"], s["args"], s["out"], s["workspace"])
    return s["out"]


def _plain_rotary(s, case):
    r, inter = case["rotary"], case["interleaved"]
    sections = _ints(case["sections"]) or [r // 2]
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device="cuda")
    freq = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    angle = s["positions"].double()[axis].t() * freq
    c, si = ((f(angle) * s["scale"]).float()[:, None] for f in (torch.cos, torch.sin))
    si = -si if case["inverse"] else si

    def turned(x):
        y = x.float()
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if inter else (y[..., :r // 2], y[..., r // 2:r])
        p, q = a * c - b * si, b * c + a * si
        head = torch.stack((p, q), -1).flatten(-2) if inter else torch.cat((p, q), -1)
        return torch.cat((head, y[..., r:]), -1).to(x.dtype)

    if not case["append"]:
        return [turned(s["q"]), turned(s["k"])]
    s["out_k"][s["out_rows"]] = turned(s["k"])
    s["out_v"][s["out_rows"]] = s["v"]
    return [turned(s["q"]), s["out_k"], s["out_v"]]


def _plain_quantize(s, case):
    n = case["rows"]

    def back(x, out):
        codes, scale, lo = _quantized(x[:n])
        half = codes.unflatten(-1, (2, x.shape[-1] // 2)).float()
        out[:n] = (lo.float().unsqueeze(-1) + scale.float().unsqueeze(-1) * half).to(x.dtype).flatten(-2)
        return out

    return [back(s["k"], s["out_k"]), back(s["v"], s["out_v"])]


def _values(codes, params, rows, values):
    """Rows of a 4-bit cache as fp32: [len(rows) ..., heads, dim]."""
    dim = 2 * codes.shape[-1]
    c, p = codes.transpose(0, 1)[rows], params.transpose(0, 1)[rows].float()
    nib = torch.stack((c & 15, c >> 4), -1).flatten(-2)[..., torch.tensor(_nibble(dim, values), device="cuda")]
    half = nib.unflatten(-1, (2, dim // 2)).float()
    return (p[..., 1::2, None] + p[..., 0::2, None] * half).flatten(-2)


def _weights(scores, visible):
    """Softmax over the visible ones; none visible: all zero."""
    scores = scores.masked_fill(~visible, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _plain_decode(s, case):
    rows = torch.tensor(_ints(case["rows"]), device="cuda")
    tails = torch.tensor(_ints(case["tails"]) or [0] * len(rows), device="cuda")
    n = rows + tails
    window, sinks = case["window"], case["sinks"]
    longest = max(r + t for r, t in zip(_ints(case["rows"]), _ints(case["tails"]) or [0] * len(rows)))
    j = torch.arange(longest if not window else min(longest, window + sinks), device="cuda")[None]
    if window:                                        # the sinks, then the last rows
        j = torch.where(j < sinks, j, j - sinks + torch.clamp(n - window, min=sinks)[:, None])
    visible = j < n[:, None]
    main = torch.clamp(torch.minimum(j, rows[:, None] - 1), min=0) + s["offsets"][:-1, None]
    main = torch.clamp(main, max=max(sum(_ints(case["rows"])) - 1, 0))
    if case["bits"] == 4:
        ck, cv, pk, pv = s["cache"]
        k, v = _values(ck, pk, main, False), _values(cv, pv, main, True)
    else:
        k, v = (x[main].float() for x in s["cache"])
    if s["tail_k"] is not None:
        late = torch.clamp(j - rows[:, None], 0, s["tail_k"].shape[1] - 1)
        b = torch.arange(len(rows), device="cuda")[:, None]
        in_tail = (j >= rows[:, None])[..., None, None]
        k = torch.where(in_tail, s["tail_k"][b, late].float(), k)
        v = torch.where(in_tail, s["tail_v"][b, late].float(), v)
    heads, dim = case["heads"], case["dim"]
    q = s["q"].float().unflatten(1, (heads, -1))                       # [batch, heads, group, dim]
    scores = q @ k.permute(0, 2, 3, 1) / math.sqrt(dim)
    out = _weights(scores, visible[:, None, None]) @ v.transpose(1, 2)
    return out.flatten(1, 2).to(s["q"].dtype)


def _plain_window(s, case):
    nq, nk = _ints(case["q_lens"]), _ints(case["k_lens"])
    heads, dim, window, sinks = case["heads"], case["dim"], case["window"], case["sinks"]
    # blocks of queries of one sequence each, and for each block the sinks and the keys from its first query's window to its last query
    blocks = [(b, i) for b, n in enumerate(nq) for i in range(0, n, _BLOCK)]
    seq = torch.tensor([b for b, _ in blocks], device="cuda")
    i = torch.tensor([x for _, x in blocks], device="cuda")[:, None] + torch.arange(_BLOCK, device="cuda")
    n_q, n_k = (torch.tensor(n, device="cuda")[seq][:, None] for n in (nq, nk))
    q0, k0 = (torch.tensor([sum(n[:b]) for b in range(len(n))], device="cuda")[seq][:, None] for n in (nq, nk))
    pos = n_k - n_q + i
    qi = q0 + torch.minimum(i, n_q - 1)
    span = min(window + _BLOCK - 1, max(nk))
    start = torch.clamp(pos[:, :1] - window + 1, min=0)
    j = torch.cat((torch.arange(sinks, device="cuda").expand(len(blocks), -1), start + torch.arange(span, device="cuda")), 1)
    near = torch.arange(sinks + span, device="cuda") >= sinks
    j3, p3 = j[:, None, :], pos[:, :, None]
    visible = (j3 <= p3) & ((j3 > p3 - window) == near) & (j3 < n_k[:, :, None])
    rows = k0 + torch.minimum(torch.clamp(j, min=0), n_k - 1)
    k, v = (x.transpose(0, 1)[:, rows].transpose(0, 1) for x in (s["k"], s["v"]))           # [blocks, heads, keys, dim]
    q = s["q"][qi].unflatten(2, (heads, -1)).permute(0, 2, 3, 1, 4)                          # [blocks, heads, group, queries, dim]
    group = q.shape[2]
    scores = (q.float().flatten(2, 3) @ k.float().transpose(2, 3) / math.sqrt(dim)).unflatten(2, (group, _BLOCK))
    w = _weights(scores, visible[:, None, None])
    out = (w.flatten(2, 3) @ v.float()).unflatten(2, (group, _BLOCK)).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return out[i < n_q].to(s["q"].dtype)


_PLAIN = dict(rotary=_plain_rotary, quantize=_plain_quantize, decode=_plain_decode, window=_plain_window)


def _pairs(nq, nk, window, sinks):
    """Visible (query, key) pairs of a sequence."""
    p = torch.arange(nk - nq, nk, dtype=torch.int64)
    seen = torch.clamp(p + 1, 0, window) + torch.clamp(torch.clamp(p - window + 1, min=0), max=sinks)
    return int(seen.sum())


def work(case):
    b, dim, heads = _BYTES[case["dtype"]], case["dim"], case["heads"]
    if case["kind"] == "rotary":
        n, axes = case["tokens"], 3 if case["sections"] else 1
        turned = n * (case["q_heads"] + heads)
        return dict(bytes=2 * turned * dim * b + (2 * n * heads * dim * b + 8 * n if case["append"] else 0) + 8 * axes * n,
                    flops=3 * turned * case["rotary"])
    if case["kind"] == "quantize":
        each = 2 * case["rows"] * heads
        return dict(bytes=each * (2 * dim * b + dim // 2 + 8), flops=4 * each * dim)
    if case["kind"] == "decode":
        rows = _ints(case["rows"])
        tails = _ints(case["tails"]) or [0] * len(rows)
        row_bytes = dim // 2 + 8 if case["bits"] == 4 else dim * b
        total = seen = 0
        for r, t in zip(rows, tails):
            first = max(0, r + t - case["window"]) if case["window"] else 0
            low = min(case["sinks"], first) if case["window"] else 0
            main = min(low, r) + max(0, r - max(first, 0))
            every = low + r + t - first
            total += main * row_bytes + (every - main) * dim * b
            seen += every
        return dict(bytes=2 * heads * total + 2 * len(rows) * case["q_heads"] * dim * b, flops=4 * dim * case["q_heads"] * seen)
    nq, nk = _ints(case["q_lens"]), _ints(case["k_lens"])
    return dict(bytes=2 * (sum(nq) * case["q_heads"] + sum(nk) * heads) * dim * b,
                flops=4 * dim * case["q_heads"] * sum(_pairs(x, y, case["window"], case["sinks"]) for x, y in zip(nq, nk)))


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    return _EXACT[case["kind"]](case, _inputs_only(case, seed))


def _inputs_only(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_rotary(case, s):
    """Every pair as a complex number times exp(i * angle)."""
    r = case["rotary"]
    axis = [a for a, n in enumerate(_ints(case["sections"]) or [r // 2]) for _ in range(n)]
    turns = torch.stack([s["positions"][axis[j]].double() * s["freq"][j] for j in range(r // 2)], 1)
    unit = torch.polar(torch.full_like(turns, s["scale"]), -turns if case["inverse"] else turns)
    first = [2 * j if case["interleaved"] else j for j in range(r // 2)]
    second = [2 * j + 1 if case["interleaved"] else j + r // 2 for j in range(r // 2)]

    def turned(x):
        y = x.double()
        z = torch.complex(y[:, :, first], y[:, :, second]) * unit.unsqueeze(1)
        y[:, :, first], y[:, :, second] = z.real, z.imag
        return y

    q, k = turned(s["q"]), turned(s["k"])
    if not case["append"]:
        return [q, k]
    ok, ov = (s[x].double() for x in ("out_k", "out_v"))
    for t, at in enumerate(s["out_rows"].tolist()):
        ok[at], ov[at] = k[t], s["v"][t].double()
    return [q, ok, ov]


def _exact_quantize(case, s):
    """The scale as a whole number of the type's steps, rounded up; the code as the nearest whole number, the even one of two."""
    digits, least = (8, -133) if case["dtype"] == "bf16" else (11, -24)
    out = []
    for name in ("k", "v"):
        x, y = s[name].double(), torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
        n, d = case["rows"], case["dim"]
        for half in (slice(0, d // 2), slice(d // 2, d)):
            part = x[:n, :, half]
            lo = part.min(dim=-1, keepdim=True).values
            want = (part.max(dim=-1, keepdim=True).values - lo) / 15
            unit = torch.exp2(torch.clamp(torch.frexp(want)[1] - digits, min=least).double())
            scale = torch.ceil(want / unit) * unit
            t = torch.where(scale > 0, (part - lo) / torch.clamp(scale, min=1e-300), torch.zeros_like(part))
            down = torch.floor(t)
            up = (t - down > 0.5) | ((t - down == 0.5) & (down % 2 == 1))
            y[:n, :, half] = lo + scale * (down + up)
        out.append(y)
    return out


def _exact_values(codes, params, values):
    """[rows, heads, dim] in 64 bits, channel by channel."""
    dim = 2 * codes.shape[2]
    out = torch.empty((codes.shape[1], codes.shape[0], dim), dtype=torch.float64, device="cuda")
    p = params.double()
    for c in range(dim):
        at = _nibble(dim, values)[c]
        code = (codes[:, :, at // 2] >> (4 * (at % 2))) & 15
        scale, lo = (p[:, :, 2 * (c >= dim // 2) + e] for e in (0, 1))
        out[:, :, c] = (lo + scale * code).t()
    return out


def _softmax_rows(scores):
    e = torch.exp(scores - scores.max(dim=-1, keepdim=True).values)
    return e / e.sum(dim=-1, keepdim=True)


def _exact_decode(case, s):
    rows = _ints(case["rows"])
    tails = _ints(case["tails"]) or [0] * len(rows)
    heads, dim = case["heads"], case["dim"]
    if case["bits"] == 4:
        ck, cv, pk, pv = s["cache"]
        mk, mv = _exact_values(ck, pk, False), _exact_values(cv, pv, True)
    else:
        mk, mv = (x.double() for x in s["cache"])
    out = torch.zeros((len(rows), case["q_heads"], dim), dtype=torch.float64, device="cuda")
    at = 0
    for b, (r, t) in enumerate(zip(rows, tails)):
        k, v = mk[at:at + r], mv[at:at + r]
        at += r
        if t:
            k, v = torch.cat((k, s["tail_k"][b, :t].double())), torch.cat((v, s["tail_v"][b, :t].double()))
        n = r + t
        if case["window"] and n > case["window"]:
            keep = [x for x in range(min(case["sinks"], n - case["window"]))] + list(range(n - case["window"], n))
            k, v = k[keep], v[keep]
        if n == 0:
            continue
        group = case["q_heads"] // heads
        for h in range(heads):
            mine = slice(h * group, (h + 1) * group)
            out[b, mine] = _softmax_rows(s["q"][b, mine].double() @ k[:, h].t() / dim ** 0.5) @ v[:, h]
    return out


def _exact_window(case, s):
    nq, nk = _ints(case["q_lens"]), _ints(case["k_lens"])
    heads, dim, window, sinks = case["heads"], case["dim"], case["window"], case["sinks"]
    group = case["q_heads"] // heads
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    q0 = k0 = 0
    for n, m in zip(nq, nk):
        for i in range(0, n, 1024):
            end = min(n, i + 1024)
            p = torch.arange(m - n + i, m - n + end, device="cuda")
            low, high = max(0, m - n + i - window + 1), m - n + end
            keys = torch.tensor([x for x in range(min(sinks, low))] + list(range(low, max(high, low))), dtype=torch.int64, device="cuda")
            if high <= 0:
                continue
            gap = p[:, None] - keys[None, :]
            seen = (gap >= 0) & ((gap < window) | (keys[None, :] < sinks))
            some = seen.any(1)
            for h in range(heads):
                k, v = s["k"][k0 + keys, h].double(), s["v"][k0 + keys, h].double()
                for j in range(h * group, (h + 1) * group):
                    x = s["q"][q0 + i:q0 + end, j].double() @ k.t() / dim ** 0.5
                    x = x.masked_fill(~seen, float("-inf"))
                    out[q0 + i:q0 + end, j] = torch.where(some[:, None], _softmax_rows(x.masked_fill(~some[:, None], 0.0)) @ v, 0.0)
        q0, k0 = q0 + n, k0 + m
    return out


_EXACT = dict(rotary=_exact_rotary, quantize=_exact_quantize, decode=_exact_decode, window=_exact_window)
