"""Mixing the tokens of many streams in few bits and constant memory, as cases that can be timed and compared.

A case is a dict of plain values; `op` says which operator it stands for:

  project  rows times a matrix of 8-bit weights: rows are taken to 8 bits with a scale each, columns of the result have one each
  append   keys, normalised and turned by position, and values into the streams' rings of 4-bit blocks
  attend   attention over a sliding window and a few first tokens that such rings hold
  scan     a gated recurrence per channel: segments of tokens, or single tokens, from a state and into one; `train`: with its gradients

Where `own` is false `run` computes the plain form in elementary torch operations; where it is true it calls the package.

A block of 4 bits is 32 neighbouring values of a head and one power of two 2^e, held as the byte e + 127 (255: the block is not a number).  A value is
a sign (bit 3) and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e; the even one of two neighbours lies in the low bits of a byte.  e is the smallest with
all of the block at most 7 * 2^e, between -100 and 125; values go to the nearest one there is, halfway to the one of even bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32
GATE = 87.0                  # gates are held to +-GATE: neither what is kept nor what is taken in is ever nothing


def listed():
    return [
        # one new row of each of 64 streams to queries, keys and values: the weights are most of what is read
        dict(name="project_rows_64", op="project", rows=64, cols=4096, outs=6144, bias=False, dtype="bf16"),
        # the rows of a push of many streams, sizes that fit no tile, float32
        dict(name="project_odd_f32", op="project", rows=777, cols=1096, outs=2001, bias=True, dtype="f32"),
        # a long prompt
        dict(name="project_prompt", op="project", rows=16384, cols=4096, outs=6144, bias=True, dtype="bf16"),
        # one new token of each of 64 streams, far into them: latency counts
        dict(name="append_step_64", op="append", streams=64, tokens=1, ragged=False, start=1 << 20, heads=8, dim=128, rotary=128, layout="half",
             slots=260, sinks=4, weight=True, stretch=1.0, dtype="bf16"),
        # pieces of prompts of uneven lengths, each on behind what its ring holds
        dict(name="append_prompt", op="append", streams=8, tokens=4096, ragged=True, start=1 << 16, heads=8, dim=128, rotary=64, layout="interleaved",
             slots=4100, sinks=4, weight=True, stretch=8.0, dtype="bf16"),
        # serving 64 streams, a token each, rings full
        dict(name="attend_step_64", op="attend", streams=64, tokens=1, ragged=False, start=1 << 20, room=0, q_heads=32, kv_heads=8, dim=128,
             window=4096, sinks=4, dtype="bf16"),
        # one stream with a wide window: few rows, a long axis
        dict(name="attend_step_1", op="attend", streams=1, tokens=1, ragged=False, start=1 << 33, room=0, q_heads=32, kv_heads=8, dim=128,
             window=65536, sinks=64, dtype="bf16"),
        # 64 live signals that bring up to 16 tokens at a time, float32
        dict(name="attend_rows_f32", op="attend", streams=64, tokens=16, ragged=True, start=5000, room=16, q_heads=8, kv_heads=4, dim=64,
             window=1000, sinks=1, dtype="f32"),
        # two long pieces of prompts
        dict(name="attend_prompt", op="attend", streams=2, tokens=8192, ragged=False, start=8192, room=8192, q_heads=32, kv_heads=8, dim=128,
             window=4096, sinks=4, dtype="bf16"),
        # one very long prompt
        dict(name="scan_prompt", op="scan", streams=1, tokens=65536, ragged=False, channels=2048, train=False, dtype="bf16"),
        # training on pieces of uneven lengths
        dict(name="scan_train", op="scan", streams=16, tokens=2048, ragged=True, channels=1536, train=True, dtype="bf16"),
        # training on short pieces of 64 live signals, channels that fill no vector, float32
        dict(name="scan_train_f32", op="scan", streams=64, tokens=48, ragged=True, channels=321, train=True, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["project", "append", "attend", "attend", "scan", "scan"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "project":
        c = dict(op=op, rows=_log(rng, 1, 16384), cols=_log(rng, 33, 8192), outs=_log(rng, 17, 8192), bias=rng.random() < 0.5, dtype=dtype)
        if rng.random() < 0.5:
            c["cols"], c["outs"] = max(64, c["cols"] // 64 * 64), max(64, c["outs"] // 64 * 64)
        while c["rows"] * c["cols"] * c["outs"] > 16384 * 4096 * 6144:
            c["rows"] = c["rows"] * 3 // 4
        return c
    if op == "append":
        step = rng.random() < 0.5
        tokens, dim = (1 if step else _log(rng, 2, 4096)), rng.choice([32, 64, 96, 128, 256])
        c = dict(op=op, streams=_log(rng, 1, 64), tokens=tokens, ragged=not step and rng.random() < 0.5, start=rng.choice([0, _log(rng, 1, 1 << 30)]),
                 heads=rng.choice([1, 2, 3, 4, 8]), dim=dim, rotary=rng.choice([0, dim // 2, dim]), layout=rng.choice(["half", "interleaved"]),
                 slots=max(64, tokens // 2) + _log(rng, 1, 512), sinks=rng.choice([0, 1, 4, 31]), weight=rng.random() < 0.5,
                 stretch=rng.choice([1.0, 4.0, 16.0]), dtype=dtype)
        while c["streams"] > 1 and c["streams"] * max(c["tokens"], c["slots"]) * c["heads"] * dim > 8 * 4096 * 8 * 128 // (2 if dtype == "f32" else 1):
            c["streams"] //= 2
        return c
    if op == "attend":
        kind = rng.choice(["step", "step", "rows", "prompt"])
        kv_heads, group, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 96, 128, 256])
        streams = _log(rng, 1, 64) if kind != "prompt" else _log(rng, 1, 8)
        tokens = {"step": 1, "rows": _log(rng, 2, 64), "prompt": _log(rng, 100, 8192)}[kind]
        c = dict(op=op, streams=streams, tokens=tokens, ragged=kind != "step" and rng.random() < 0.5, start=rng.choice([0, _log(rng, 1, 1 << 34)]),
                 room=rng.choice([tokens - 1, tokens + 40]), q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim, window=_log(rng, 16, 65536),
                 sinks=rng.choice([0, 1, 4, 31]), dtype=dtype)
        most = work(next(x for x in listed() if x["name"] == "attend_prompt"))["flops"] / (8 if dtype == "f32" else 2)
        while work(c)["flops"] > most or c["streams"] * (c["window"] + c["room"]) * kv_heads * dim > 64 * 4100 * 8 * 128:
            if c["tokens"] > 64:
                c["room"] -= c["tokens"] - c["tokens"] // 2
                c["tokens"] //= 2
            elif c["streams"] > 1:
                c["streams"] //= 2
            else:
                c["window"] //= 2
        return c
    kind = rng.choice(["step", "rows", "prompt", "prompt"])
    c = dict(op=op, streams=_log(rng, 1, 64), tokens={"step": 1, "rows": _log(rng, 2, 64), "prompt": _log(rng, 100, 65536)}[kind],
             ragged=kind != "step" and rng.random() < 0.5, channels=_log(rng, 33, 4096), train=kind != "step" and rng.random() < 0.6, dtype=dtype)
    if rng.random() < 0.5:
        c["channels"] = max(64, c["channels"] // 64 * 64)
    while c["streams"] * c["tokens"] * c["channels"] * (4 if c["train"] else 1) * (2 if dtype == "f32" else 1) > 65536 * 2048:
        if c["streams"] > 1:
            c["streams"] //= 2
        else:
            c["tokens"] //= 2
    return c


def _lengths(case):
    """Tokens of each segment: uneven ones where the case says so, a whole one and one without any among them."""
    if not case["ragged"]:
        return [case["tokens"]] * case["streams"]
    n = [1 + int(case["tokens"] * (0.618034 * i % 1)) for i in range(case["streams"])]
    n[0] = case["tokens"]
    if case["streams"] > 2:
        n[1] = 0
    return n


def _frequencies(case):
    """Radians per position of each pair, in 64 bits: slow ones are stretched, quick ones are not, with a ramp between."""
    half = case["rotary"] // 2
    i = torch.arange(half, dtype=torch.float64)
    f = 10000.0 ** (-i / max(half, 1))
    turns = f * 4096 / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    return f * keep + f / case["stretch"] * (1 - keep)


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    t = DTYPE[case["dtype"]]

    def normal(*shape, dtype=t):
        return torch.randn(shape, device=DEVICE, generator=g).to(dtype)

    def blocks(streams, heads, slots, dim):
        """Any codes, with powers of two as keys and values of a few units have them."""
        codes = torch.randint(0, 256, (streams, heads, slots, dim // 2), device=DEVICE, generator=g, dtype=torch.uint8)
        return codes, torch.randint(124, 127, (streams, heads, slots, dim // BLOCK), device=DEVICE, generator=g, dtype=torch.uint8)
    s = dict(case=case)
    if case["op"] == "project":
        rows, cols, outs = case["rows"], case["cols"], case["outs"]
        padded = -(-cols // 16) * 16               # rows of codes are filled up to 16 with zeros
        s["x"] = normal(rows, cols) * torch.exp(0.5 * normal(rows, 1))
        s["weight"] = torch.zeros(outs, padded, dtype=torch.int8, device=DEVICE)
        s["weight"][:, :cols] = (40 * torch.randn(outs, cols, device=DEVICE, generator=g)).round_().clamp_(-127, 127).to(torch.int8)
        s["weight_scales"] = torch.exp(0.2 * normal(outs, dtype=torch.float32)) / (40 * math.sqrt(cols))
        s["bias"] = normal(outs, dtype=torch.float32) if case["bias"] else None
        return s
    n = _lengths(case)
    total, streams = sum(n), case["streams"]
    s["offsets"] = None
    if case["ragged"]:
        s["offsets"] = torch.tensor([0] + n).cumsum(0).to(DEVICE)
        s["max_tokens"] = max(n)
    if case["op"] == "scan":
        c = case["channels"]
        s["x"] = normal(total, c)
        # gates that keep anything between a few tokens and a few thousand
        s["gates"] = normal(total, c) + (1 + 6 * torch.rand(c, device=DEVICE, generator=g)).to(t)
        s["state"], s["state_out"] = normal(streams, c, dtype=torch.float32), torch.empty(streams, c, device=DEVICE)
        if case["train"]:
            s["grad"], s["grad_end"] = normal(total, c), normal(streams, c, dtype=torch.float32)
        return s
    s["starts"] = torch.randint(case["start"] // 2, case["start"] + 1, (streams,), device=DEVICE, generator=g)
    d = case["dim"]
    if case["op"] == "append":
        heads = case["heads"]
        # what a projection leaves: keys and values lie next to each other in a token's row
        packed = normal(total, 2 * heads * d) * 1.5
        s["k"], s["v"] = packed[:, :heads * d].unflatten(1, (heads, d)), packed[:, heads * d:].unflatten(1, (heads, d))
        s["ring"] = blocks(streams, heads, case["slots"], d) + blocks(streams, heads, case["slots"], d)
        s["frequencies"] = _frequencies(case).to(DEVICE)
        s["amplitude"] = 0.1 * math.log(case["stretch"]) + 1.0
        s["k_weight"] = 1 + 0.2 * torch.randn(d, device=DEVICE, generator=g) if case["weight"] else None
        return s
    heads, slots = case["kv_heads"], case["sinks"] + case["window"] + case["room"]
    s["q"] = normal(total, case["q_heads"], d)
    # every slot holds something: rows that the stream has not written yet are what another left there
    s["ring"] = blocks(streams, heads, slots, d) + blocks(streams, heads, slots, d)
    return s


def run(state):
    if own:
        return _run_own(state)
    return {"project": _project, "append": _append, "attend": _attend, "scan": _scan}[state["case"]["op"]](state)


def _run_own(s):
    import paper_1804_10727_amd as idf
    c = s["case"]
    if c["op"] == "project":
        return idf.project_rows(s["x"], s["weight"], s["weight_scales"], bias=s["bias"])
    ragged = {} if s["offsets"] is None else dict(offsets=s["offsets"], max_tokens=s["max_tokens"])
    if c["op"] == "append":
        ring = idf.NibbleRing(*s["ring"])
        idf.nibble_append(s["k"], s["v"], ring, s["starts"], sinks=c["sinks"], frequencies=s["frequencies"], layout=c["layout"],
                         amplitude=s["amplitude"], k_weight=s["k_weight"], eps=1e-6, **ragged)
        return idf.nibble_values(ring)
    if c["op"] == "attend":
        return idf.nibble_attend(s["q"], idf.NibbleRing(*s["ring"]), s["starts"], window=c["window"], sinks=c["sinks"], **ragged)
    if not c["train"]:
        return idf.gate_scan(s["x"], s["gates"], state=s["state"], state_out=s["state_out"], **ragged), s["state_out"]
    # as a training program has them: leaves that record, a forward and a backward pass
    x, gates, state = (s[k].detach().requires_grad_() for k in ("x", "gates", "state"))
    out, end = idf.gate_scan_recorded(x, gates, state, **ragged)
    return out.detach(), end.detach(), *torch.autograd.grad((out, end), (x, gates, state), (s["grad"], s["grad_end"]))


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ----

def _project(s):
    x = s["x"].double()
    most = x.abs().amax(1, keepdim=True)
    # in 64 bits: next to the middle between two codes 32 would not do (127 x is exact there, and no quotient that is not the middle rounds to it)
    codes = torch.round(x * 127 / most.clamp(min=1e-300)).float()
    scale = (most / 127).float()
    out = (codes @ s["weight"][:, :s["case"]["cols"]].float().T) * scale * s["weight_scales"]
    return (out if s["bias"] is None else out + s["bias"]).to(s["x"].dtype)


def _token_places(s):
    """Of every packed token its segment, and its place in it."""
    c, n = s["case"], s["k" if s["case"]["op"] == "append" else "x" if s["case"]["op"] == "scan" else "q"].shape[0]
    i = torch.arange(n, device=DEVICE)
    if s["offsets"] is None:
        return i // c["tokens"], i % c["tokens"]
    segment = torch.searchsorted(s["offsets"], i, right=True) - 1
    return segment, i - s["offsets"][segment]


def _to_blocks(y):
    """[..., dim] in 64 bits: codes [..., dim / 2] and powers [..., dim / 32]."""
    y = y.unflatten(-1, (-1, BLOCK))
    most = y.abs().amax(-1)
    mantissa, power = torch.frexp(most)
    e = torch.where(mantissa <= 0.875, power - 3, power - 2).clamp(-100, 125)
    e = torch.where(most == 0, -100, e)
    y = torch.ldexp(y, -e[..., None])
    size = y.abs()
    # steps of 0.5 up to 2, of 1 up to 4, then 2
    code = torch.where(size < 1.75, torch.round(2 * size), torch.where(size < 3.5, 2 + torch.round(size), 4 + torch.round(size / 2).clamp(max=3)))
    code = code.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    code = code.flatten(-2)
    fine = torch.isfinite(most)
    scale = torch.where(fine, e + 127, 255).to(torch.uint8)
    return torch.where(fine.repeat_interleave(BLOCK // 2, -1), code[..., 0::2] | (code[..., 1::2] << 4), 0), scale


def _from_blocks(codes, scales):
    """The values that blocks stand for, in 32 bits."""
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEVICE)
    y = torch.stack([levels[(codes & 15).int()], levels[(codes >> 4).int()]], -1).flatten(-2)
    e = scales.float() - 127
    return (y.unflatten(-1, (-1, BLOCK)) * torch.where(scales == 255, math.nan, torch.exp2(e))[..., None]).flatten(-2)


def _slot(p, sinks, slots):
    return torch.where(p < sinks, p, sinks + (p - sinks) % (slots - sinks))


def _append(s):
    c = s["case"]
    r = c["rotary"]
    segment, t = _token_places(s)
    p = s["starts"][segment] + t
    y = s["k"].double()                            # (codes next to the middle between two: 32 bits would not do)
    if s["k_weight"] is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * s["k_weight"].double()
    if r:
        angle = p.double()[:, None] * s["frequencies"]
        cos, sin = ((f(angle) * s["amplitude"])[:, None, :] for f in (torch.cos, torch.sin))
        a, b = (y[..., :r // 2], y[..., r // 2:r]) if c["layout"] == "half" else (y[..., 0:r:2], y[..., 1:r:2])
        turned = [a * cos - b * sin, b * cos + a * sin]
        y = torch.cat([torch.cat(turned, -1) if c["layout"] == "half" else torch.stack(turned, -1).flatten(-2), y[..., r:]], -1)
    lengths = s["offsets"].diff() if s["offsets"] is not None else torch.full((c["streams"],), c["tokens"], device=DEVICE)
    # the newest rows that the ring has room for, and the first tokens
    keep = (p < c["sinks"]) | (t >= lengths[segment] - (c["slots"] - c["sinks"]))
    stream, where = segment[keep], _slot(p, c["sinks"], c["slots"])[keep]
    for new, codes, scales in ((y, s["ring"][0], s["ring"][1]), (s["v"].double(), s["ring"][2], s["ring"][3])):
        codes_, scales_ = _to_blocks(new[keep])
        codes[stream, :, where], scales[stream, :, where] = codes_, scales_
    return tuple(_from_blocks(*s["ring"][i:i + 2]).to(torch.bfloat16).transpose(1, 2).contiguous() for i in (0, 2))


def _attend(s):
    c = s["case"]
    window, sinks, dim, hkv, streams = c["window"], c["sinks"], c["dim"], c["kv_heads"], c["streams"]
    slots, group = s["ring"][0].shape[2], c["q_heads"] // c["kv_heads"]
    q, start = s["q"], s["starts"][:, None]
    longest = s.get("max_tokens", c["tokens"])
    if s["offsets"] is not None:                   # [streams][longest]: where each of them lies, and whether it is one
        t = torch.arange(longest, device=DEVICE)[None, :]
        there = t < s["offsets"].diff()[:, None]
        q = q[(s["offsets"][:-1, None] + t).clamp(0, q.shape[0] - 1)]
    else:
        there, q = None, q.unflatten(0, (streams, longest))
    # rings of a part of the streams at a time, in 32 bits
    some = max(1, min(streams, int(4e9) // (slots * hkv * dim * 4)))
    outs = []
    for b in range(0, streams, some):
        k, v = (_from_blocks(s["ring"][i][b:b + some], s["ring"][i + 1][b:b + some]) for i in (0, 2))
        n, row = k.shape[0], torch.arange(k.shape[0], device=DEVICE)[:, None]
        step = max(1, min(longest, 512, int(1.5e9) // (n * c["q_heads"] * min(window + 512, window + longest))))
        parts = []
        for at in range(0, longest, step):
            m = min(step, longest - at)
            p = start[b:b + some] + at + torch.arange(m, device=DEVICE)[None, :]
            first = torch.arange(sinks, device=DEVICE)[None, :].expand(n, -1)
            j = torch.cat([first, p[:, :1] - window + 1 + torch.arange(window + m - 1, device=DEVICE)[None, :]], 1)
            is_first = torch.arange(j.shape[1], device=DEVICE) < sinks
            seen = is_first | (j >= sinks)
            pos, ask = j[:, None, :], p[:, :, None]
            visible = seen[:, None, :] & (pos >= 0) & (pos <= ask) & (is_first | (pos > ask - window))
            place = _slot(j.clamp(min=0), sinks, slots)[:, None, :].expand(-1, hkv, -1)
            head = torch.arange(hkv, device=DEVICE)[None, :, None]
            kk, vv = (x[row[:, :, None], head, place] for x in (k, v))                           # [streams][heads][keys][dim]
            qq = q[b:b + some, at:at + m].float().unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).reshape(n, hkv, group * m, dim)
            score = (qq @ kk.transpose(2, 3).contiguous() / math.sqrt(dim)).unflatten(2, (group, m))
            score = score.masked_fill_(~visible[:, None, None], -math.inf)
            score = torch.exp(score - score.amax(-1, keepdim=True))
            o = (score.flatten(2, 3) @ vv).unflatten(2, (group, m)) / score.sum(-1, keepdim=True)
            parts.append(o.permute(0, 3, 1, 2, 4).flatten(2, 3))
        outs.append(torch.cat(parts, 1))
    out = torch.cat(outs).to(s["q"].dtype)
    return out[there] if there is not None else out.flatten(0, 1)


def _recurrence(keep, new):
    """y_t = keep_t y_{t-1} + new_t along the first axis, by doubling."""
    shift = 1
    while shift < keep.shape[0]:
        new = torch.cat([new[:shift], torch.addcmul(new[shift:], keep[shift:], new[:-shift])])
        keep = torch.cat([keep[:shift], keep[shift:] * keep[:-shift]])
        shift *= 2
    return new


def _scan(s):
    c = s["case"]
    t = s["x"].dtype
    x, g = s["x"].float(), s["gates"].float().clamp(-GATE, GATE)
    keep, take = torch.sigmoid(g), torch.sigmoid(-g)
    segment, place = _token_places(s)
    lengths = s["offsets"].diff() if s["offsets"] is not None else torch.full((c["streams"],), c["tokens"], device=DEVICE)
    first, last = (place == 0)[:, None], (place == lengths[segment] - 1)[:, None]
    some = (lengths > 0)[:, None]
    begins = lengths.cumsum(0) - lengths
    at_first, at_last = ((i.clamp(0, x.shape[0] - 1)) for i in (begins, begins + lengths - 1))
    # a segment's first token takes the state in, and nothing is kept of the tokens in front of it
    before = s["state"][segment]
    h = _recurrence(torch.where(first, 0, keep), torch.addcmul(take * x, keep * first, before))
    end = torch.where(some, h[at_last], s["state"])
    if not c["train"]:
        s["state_out"].copy_(end)
        return h.to(t), s["state_out"]
    behind = torch.cat([keep[1:], keep[:1]])       # what the next token keeps
    dh = torch.addcmul(s["grad"].float(), last.float(), s["grad_end"][segment])
    dh = _recurrence(torch.where(last, 0, behind).flip(0), dh.flip(0)).flip(0)
    was = torch.where(first, before, torch.cat([h[:1], h[:-1]]))
    return h.to(t), end, (dh * take).to(t), (dh * (was - x) * keep * take).to(t), torch.where(some, (dh * keep)[at_first], s["grad_end"])


# ---- the definitions in 64 bits ----

def _exact_values(y):
    """What a block of 4 bits holds of each value: the nearest level, by the borders between them."""
    y = y.unflatten(-1, (-1, BLOCK))
    most = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -100)
    for power in range(-100, 125):
        e += (most > 7 * 2.0 ** power).double()
    size = y.abs() * torch.exp2(-e)
    levels, at = torch.tensor(LEVELS, device=DEVICE, dtype=torch.float64), torch.zeros(y.shape, dtype=torch.long, device=DEVICE)
    for i in range(7):
        border = (LEVELS[i] + LEVELS[i + 1]) / 2
        at += (size >= border) if i % 2 else (size > border)
    return (torch.copysign(levels[at], y) * torch.exp2(e)).flatten(-2)


def _exact_held(codes, scales):
    y = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=DEVICE)
    for at, nibble in ((0, codes % 16), (1, codes // 16)):
        code, value = nibble % 8, torch.zeros(codes.shape, dtype=torch.float64, device=DEVICE)
        for i, level in enumerate(LEVELS):
            value[code == i] = level
        y[..., at::2] = torch.where(nibble >= 8, -value, value)
    return y * torch.pow(2.0, scales.double() - 127).repeat_interleave(BLOCK, -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "project":
        out = torch.empty(case["rows"], case["outs"], dtype=torch.float64, device=DEVICE)
        w = s["weight"][:, :case["cols"]].double() * s["weight_scales"].double()[:, None]
        for lo in range(0, case["rows"], 2048):
            x = s["x"][lo:lo + 2048].double()
            scale = x.abs().max(1, keepdim=True).values
            out[lo:lo + 2048] = (torch.round(127 * x / scale) * (scale / 127)) @ w.T
        return out if s["bias"] is None else out + s["bias"].double()
    n, first = _lengths(case), 0
    if case["op"] == "append":
        held = [_exact_held(*s["ring"][i:i + 2]).transpose(1, 2).contiguous() for i in (0, 2)]
        r, sinks, period = case["rotary"], case["sinks"], case["slots"] - case["sinks"]
        for b, start in enumerate(s["starts"].tolist()):
            new = [t for t in range(n[b]) if start + t < sinks or t >= n[b] - period]
            at = torch.tensor([start + t if start + t < sinks else sinks + (start + t - sinks) % period for t in new], dtype=torch.long, device=DEVICE)
            t = torch.tensor(new, dtype=torch.long, device=DEVICE)
            y, v = s["k"][first + t].double(), s["v"][first + t].double()
            first += n[b]
            if not new:
                continue
            if s["k_weight"] is not None:
                y = s["k_weight"].double() * y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / case["dim"] + 1e-6)
            if r:
                turn = torch.polar(torch.full((len(new), r // 2), s["amplitude"], dtype=torch.float64, device=DEVICE), (start + t).double()[:, None] * s["frequencies"])
                lo, hi = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
                z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * turn[:, None]
                y[..., lo], y[..., hi] = z.real, z.imag
            held[0][b, at], held[1][b, at] = _exact_values(y), _exact_values(v)
        return tuple(held)
    if case["op"] == "attend":
        group, slots = case["q_heads"] // case["kv_heads"], s["ring"][0].shape[2]
        window, sinks, period = case["window"], case["sinks"], slots - case["sinks"]
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
        for b, start in enumerate(s["starts"].tolist()):
            keys, values = (_exact_held(s["ring"][i][b], s["ring"][i + 1][b]) for i in (0, 2))
            for lo in range(0, n[b], 2048):
                m = min(n[b] - lo, 2048)
                low, top = start + lo, start + lo + m - 1
                pos = torch.cat([torch.arange(0, min(sinks, top + 1), device=DEVICE), torch.arange(max(sinks, low - window + 1), top + 1, device=DEVICE)])
                at = torch.where(pos < sinks, pos, sinks + (pos - sinks) % period)
                p = low + torch.arange(m, device=DEVICE)
                hidden = (pos > p[:, None]) | ((pos <= p[:, None] - window) & (pos >= sinks))
                tokens = slice(first + lo, first + lo + m)
                for h in range(case["q_heads"]):
                    score = s["q"][tokens, h].double() @ keys[h // group, at].T / math.sqrt(case["dim"])
                    out[tokens, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ values[h // group, at]
            first += n[b]
        return out
    # token by token, all streams side by side
    longest, streams, c = max(n), case["streams"], case["channels"]
    begins = torch.tensor([sum(n[:b]) for b in range(streams)], device=DEVICE)
    lengths = torch.tensor(n, device=DEVICE)
    total = sum(n)
    h, was = s["state"].double(), torch.empty(total, c, dtype=torch.float64, device=DEVICE) if case["train"] else None
    out = torch.empty(total, c, dtype=torch.float64, device=DEVICE)
    x, keep = s["x"].double(), 1 / (1 + torch.exp(-s["gates"].double().clamp(-GATE, GATE)))
    even = all(m == longest for m in n)
    by = [torch.arange(streams, device=DEVICE) if even else torch.nonzero(lengths > t).flatten() for t in range(longest)]
    for t in range(longest):
        at = begins[by[t]] + t
        if case["train"]:
            was[at] = h[by[t]]
        h[by[t]] = keep[at] * h[by[t]] + (1 - keep[at]) * x[at]
        out[at] = h[by[t]]
    if not case["train"]:
        return out, h
    d, dx, dg = s["grad_end"].double(), torch.empty_like(out), torch.empty_like(out)
    for t in reversed(range(longest)):
        at = begins[by[t]] + t
        now = d[by[t]] + s["grad"][at].double()
        dx[at] = (1 - keep[at]) * now
        dg[at] = now * (was[at] - x[at]) * keep[at] * (1 - keep[at])
        d[by[t]] = now * keep[at]
    return out, h, dx, dg, d


def work(case):
    """Inputs read once and outputs written once."""
    e = BYTES[case["dtype"]]
    if case["op"] == "project":
        r, k, n = case["rows"], case["cols"], case["outs"]
        return dict(bytes=r * k * e + k * n + r * n * e + 4 * n, flops=2 * r * k * n)
    if case["op"] == "append":
        kept = sum(min(t, case["slots"] - case["sinks"]) for t in _lengths(case)) * case["heads"] * case["dim"]
        held = case["streams"] * case["slots"] * case["heads"] * case["dim"]
        # new tokens read and their blocks written; then the rings read and the values that they stand for written
        return dict(bytes=2 * kept * (e + 17 / 32) + 2 * held * (17 / 32 + 2), flops=20 * kept)
    if case["op"] == "attend":
        hq, hkv, d, window, sinks, start = case["q_heads"], case["kv_heads"], case["dim"], case["window"], case["sinks"], 0.75 * case["start"]
        nbytes = flops = 0
        for t in _lengths(case):
            held = min(start + t, window + t - 1) + (sinks if start > window else 0)       # rows of the ring that some query sees
            grow = max(0.0, min(t, window - start))                                       # queries whose window reaches the beginning
            pairs = grow * (start + (grow + 1) / 2) + (t - grow) * (window + sinks)
            nbytes += 2 * e * t * hq * d + (2 * held * hkv * d * 17 / 32 if t else 0)
            flops += pairs * hq * 4 * d
        return dict(bytes=nbytes, flops=flops)
    n, c, streams = sum(_lengths(case)), case["channels"], case["streams"]
    if not case["train"]:
        return dict(bytes=3 * n * c * e + 8 * streams * c, flops=6 * n * c)
    return dict(bytes=8 * n * c * e + 16 * streams * c, flops=20 * n * c)
