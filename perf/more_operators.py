"""Workloads of the operators around attention: rotary positions of several axes, attention of prompts over
their own 16-bit keys and values, a key/value cache in 4 bits (written and read back) and attention over it.

`run` takes one pass through an operator: in elementary torch operations in 32 bits (`own` false)
or through the library's entry points (`own` true), on the same inputs.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------- cases
def listed():
    return [
        # A decoding batch of text: one token each, the three axes at one position. Latency.
        dict(name="rotary_token", op="rotary", tokens=64, heads=32, kv_heads=8, dim=128, rotary=128,
             axes=3, pairs="halves", far=32768),
        # A two-axis image model with rotations of a part of each head, neighbours paired, odd counts.
        dict(name="rotary_odd", op="rotary", tokens=1333, heads=12, kv_heads=2, dim=64, rotary=48,
             axes=2, pairs="neighbours", far=1000),
        # A video's tokens in one prompt: time, height and width.
        dict(name="rotary_video", op="rotary", tokens=16384, heads=32, kv_heads=8, dim=128, rotary=128,
             axes=3, pairs="halves", far=8192),
        # One question of a few words: latency.
        dict(name="prompt_short", op="prompt", batch=1, heads=32, kv_heads=8, dim=128, length=77,
             causal=True, window=0),
        # Prompts of very different lengths in one call.
        dict(name="prompt_packed", op="prompt", batch=12, heads=32, kv_heads=8, dim=128, length=2048,
             causal=True, window=0),
        # One long document: bound by the tensor cores and the exponentials.
        dict(name="prompt_long", op="prompt", batch=1, heads=32, kv_heads=8, dim=128, length=8192,
             causal=True, window=0),
        # Each sequence of a batch appends one token to the cache; the block it lands in is read back.
        dict(name="cache4_token", op="cache", batch=64, heads=32, kv_heads=8, dim=128, page=16,
             past=4096, new=1, read=16),
        # A prompt is written to the cache behind a shared prefix, and everything is read back.
        dict(name="cache4_prompt", op="cache", batch=4, heads=32, kv_heads=8, dim=128, page=64,
             past=1000, new=8192, read=9192),
        # One short conversation, one token: latency.
        dict(name="attention4_short", op="attention", batch=1, heads=32, kv_heads=8, dim=128, page=16,
             length=1000, new=1, window=0),
        # A batch of conversations of very different lengths, one token each.
        dict(name="attention4_batch", op="attention", batch=64, heads=32, kv_heads=8, dim=128, page=32,
             length=8192, new=1, window=0),
        # One document of 128 K tokens, four tokens to verify, every head with its own keys.
        dict(name="attention4_long", op="attention", batch=1, heads=16, kv_heads=16, dim=64, page=64,
             length=131071, new=4, window=0),
        # A chunk of a long prompt against what is already cached.
        dict(name="attention4_chunk", op="attention", batch=2, heads=32, kv_heads=8, dim=128, page=64,
             length=8192, new=1024, window=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("rotary", "prompt", "cache", "attention"))
        kv_heads = rng.choice((1, 2, 4, 8, 16))
        c = dict(op=op, heads=kv_heads * rng.choice((1, 2, 3, 4, 8)), kv_heads=kv_heads,
                 dim=rng.choice((64, 128, 256)))
        if op == "rotary":
            c.update(tokens=_log(rng, 1, 32768), rotary=16 * rng.randint(1, c["dim"] // 16),
                     axes=rng.choice((1, 2, 3, 4)), pairs=rng.choice(("halves", "neighbours")),
                     far=_log(rng, 16, 1 << 22))
        elif op == "prompt":
            c.update(batch=_log(rng, 1, 32), length=_log(rng, 1, 8192), causal=rng.random() < 0.8)
            c["window"] = rng.choice((0, 0, _log(rng, 16, 4096))) if c["causal"] else 0
        else:
            c.update(batch=_log(rng, 1, 128), page=rng.choice((16, 32, 64, 128)))
            new = 1 if rng.random() < 0.6 else _log(rng, 2, 4096)
            if op == "cache":
                past = _log(rng, 1, 8192) - 1
                c.update(past=past, new=new, read=rng.choice((min(past + new, 64), past + new)))
            else:
                c.update(length=max(new, _log(rng, 1, 131072)), new=new,
                         window=rng.choice((0, 0, 0, _log(rng, 16, 4096))))
        if _cost(c) <= top and _plain_values(c) <= 1 << 30:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _plain_values(case):
    """Values of the largest tensor the plain form makes."""
    if case["op"] == "attention":
        most = max(case["heads"] * case["new"], case["kv_heads"] * case["dim"])
        return case["batch"] * case["length"] * most
    if case["op"] == "cache":
        return case["batch"] * (case["past"] + case["new"] + case["page"]) * case["kv_heads"] * case["dim"]
    if case["op"] == "prompt":
        return case["heads"] * min(case["length"], 512) * max(case["length"], case["dim"] * case["batch"])
    return case["tokens"] * case["heads"] * case["dim"]


def _spread(most, count, least=0):
    """`count` lengths in [least, most], spread evenly in no particular order, the first the largest."""
    return [most - int((most - least) * ((i * 0.6180339887498949) % 1.0)) for i in range(count)]


def _lengths(case):
    """Per sequence: tokens cached before the call, tokens the call adds (already in the cache for attention)."""
    b = case["batch"]
    if case["op"] == "prompt":
        return [0] * b, _spread(case["length"], b, 1)
    new = _spread(case["new"], b, 1 if case["new"] == 1 else max(1, case["new"] // 2))
    if case["op"] == "cache":
        return _spread(case["past"], b), new
    total = [max(t, n) for t, n in zip(_spread(case["length"], b, 1), new)]
    return [t - n for t, n in zip(total, new)], new


def _sections(case):
    """Frequencies of each axis: the first takes what the others leave, as time does."""
    count, axes = case["rotary"] // 2, case["axes"]
    rest = [count * 3 // (4 * axes - 1 + (axes == 1))] * (axes - 1)
    return [count - sum(rest)] + rest


def work(case):
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotary":
        values = case["tokens"] * (hq + hk) * d
        return {"bytes": 4 * values + 4 * case["tokens"] * case["axes"] + 2 * case["rotary"],
                "flops": 3.0 * case["tokens"] * (hq + hk) * case["rotary"]}
    past, new = _lengths(case)
    stored = d // 2 + 4  # of a token and head, K or V: codes, scale and offset
    if case["op"] == "cache":
        read = sum(min(case["read"], p + n) for p, n in zip(past, new))
        return {"bytes": 2 * hk * (sum(new) + read) * (stored + 2 * d), "flops": 0.0}
    pairs = seen = 0
    for p, n in zip(past, new):
        if not case.get("causal", True):
            pairs += n * n
            continue
        w = case["window"] or (p + n)
        seen += min(p + n, n - 1 + w)
        # query i at position p + i sees min(p + i + 1, w) tokens
        full = max(0, min(n, w - p - 1))
        pairs += full * (p + 1) + full * (full - 1) // 2 + (n - full) * min(w, p + n)
    by = 2 * 2 * sum(new) * hq * d
    by += 2 * 2 * sum(new) * hk * d if case["op"] == "prompt" else 2 * hk * seen * stored
    return {"bytes": by, "flops": 4.0 * pairs * hq * d}


# --------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def starts(counts):
        return ints([sum(counts[:i]) for i in range(len(counts) + 1)])

    s = dict(case)
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotary":
        past, new = None, [case["tokens"]]
    else:
        past, new = _lengths(case)
    # queries, keys and values of the new tokens as one projection leaves them: one row per token
    qkv = normal(sum(new), (hq + 2 * hk) * d).half()
    s["q"] = qkv[:, : hq * d].view(-1, hq, d)
    s["k_new"] = qkv[:, hq * d: (hq + hk) * d].view(-1, hk, d)
    s["v_new"] = qkv[:, (hq + hk) * d:].view(-1, hk, d)
    if case["op"] == "rotary":
        s["sections"] = _sections(case)
        s["positions"] = (uniform(case["axes"], case["tokens"]) * case["far"]).to(torch.int32)
        r = case["rotary"]
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)).float()
        return s
    s["cu_new"], s["max_new"] = starts(new), max(new)
    s["softmax_scale"] = 1.0 / math.sqrt(d)
    if case["op"] == "prompt":
        s["lengths"] = new
        return s
    b, page = case["batch"], case["page"]
    pages = [-(-(p + n) // page) for p, n in zip(past, new)]
    total = sum(pages) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((b, max(pages)), dtype=torch.int32, device="cuda")
    valid = torch.arange(max(pages), device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    table[valid] = order[: sum(pages)]
    s["table"], s["spare"] = table, order[-1].long()
    for name in ("k", "v"):
        s[name + "_cache"] = torch.randint(0, 256, (total, hk, page, d // 2), generator=g, device="cuda",
                                           dtype=torch.uint8)
        step = 0.25 + 0.2 * uniform(total, hk, page)
        s[name + "_scale"] = torch.stack((step, -step * (6.5 + 2.0 * uniform(total, hk, page))), dim=3).half()
    s["past"] = ints(past)
    s["total"] = ints([p + n for p, n in zip(past, new)])
    s["max_total"] = max(p + n for p, n in zip(past, new))
    if case["op"] == "cache":
        read = [min(case["read"], p + n) for p, n in zip(past, new)]
        s["cu_read"], s["max_read"], s["tokens_read"] = starts(read), max(read), sum(read)
        s["first_read"] = ints([p + n - r for p, n, r in zip(past, new, read)])
    return s


# ------------------------------------------------------------------------------- plain form
def _plain_rotary(s):
    r, count = s["rotary"], s["rotary"] // 2
    axis = torch.repeat_interleave(torch.arange(s["axes"], device="cuda"),
                                   torch.tensor(s["sections"], device="cuda"), output_size=count)
    angle = s["positions"][axis].double().t() * s["inv_freq"].double()  # [tokens, count]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    outs = []
    for name in ("q", "k_new"):
        x = s[name].float()
        y = x.clone()
        if s["pairs"] == "halves":
            first, second = slice(0, count), slice(count, r)
        else:
            first, second = slice(0, r, 2), slice(1, r, 2)
        a, b = x[..., first], x[..., second]
        y[..., first] = a * cos - b * sin
        y[..., second] = b * cos + a * sin
        outs.append(y.half())
    return outs


def _plain_prompt(s):
    hq, hk, d = s["heads"], s["kv_heads"], s["dim"]
    out, at = torch.empty_like(s["q"], memory_format=torch.contiguous_format), 0
    for n in s["lengths"]:
        k, v = (s[name][at: at + n].float().transpose(0, 1) for name in ("k_new", "v_new"))
        for lo in range(0, n, 512):
            hi = min(n, lo + 512)
            end = hi if s["causal"] else n
            begin = max(0, lo - s["window"] + 1) if s["window"] else 0
            q = s["q"][at + lo: at + hi].float().view(hi - lo, hk, hq // hk, d).permute(1, 2, 0, 3)
            scores = q.reshape(hk, -1, d) @ k[:, begin:end].transpose(1, 2) * s["softmax_scale"]
            scores = scores.view(hk, hq // hk, hi - lo, end - begin)
            if s["causal"]:
                place = torch.arange(lo, hi, device="cuda")[:, None]
                token = torch.arange(begin, end, device="cuda")[None, :]
                hidden = token > place
                if s["window"]:
                    hidden = hidden | (token <= place - s["window"])
                scores = scores.masked_fill(hidden, -math.inf)
            weights = torch.exp(scores - scores.amax(3, keepdim=True))
            o = (weights.view(hk, -1, end - begin) @ v[:, begin:end]).view(hk, hq // hk, hi - lo, d)
            o = o / weights.sum(3, keepdim=True)
            out[at + lo: at + hi] = o.permute(2, 0, 1, 3).reshape(hi - lo, hq, d).half()
        at += n
    return out


def _packed(cu, tokens):
    """Per row of the packed order: its sequence and its place among that sequence's rows."""
    seq = torch.repeat_interleave(torch.arange(cu.shape[0] - 1, device="cuda"), cu[1:] - cu[:-1],
                                  output_size=tokens)
    return seq, torch.arange(tokens, device="cuda") - cu[seq]


def _plain_append(s, name):
    x = s[name + "_new"].float()
    least, most = x.amin(2), x.amax(2)
    step = ((most - least) / torch.full_like(most, 15.0)).half()  # (a tensor: division by a number is a product)
    inverse = torch.where(step > 0, torch.ones_like(most) / step.float(), torch.zeros_like(most))
    code = torch.round((x - least[..., None]) * inverse[..., None]).clamp(0, 15).to(torch.uint8)
    code = code[..., 0::2] | (code[..., 1::2] << 4)
    seq, place = _packed(s["cu_new"], x.shape[0])
    at = s["past"][seq] + place
    slot, row = s["table"][seq, at // s["page"]].long(), (at % s["page"]).long()
    s[name + "_cache"][slot, :, row] = code
    s[name + "_scale"][slot, :, row] = torch.stack((step, least.half()), dim=2)


def _values(code, scale):
    """Codes [..., dim / 2] and (scale, offset) [..., 2] as FP32 values [..., dim]."""
    code = torch.stack((code & 15, code >> 4), dim=-1).flatten(-2).float()
    scale = scale.float()
    return scale[..., 1:] + code * scale[..., :1]


def _plain_read(s, name):
    seq, place = _packed(s["cu_read"], s["tokens_read"])
    at = s["first_read"][seq] + place
    slot, row = s["table"][seq, at // s["page"]].long(), (at % s["page"]).long()
    return _values(s[name + "_cache"][slot, :, row], s[name + "_scale"][slot, :, row]).half()


def _plain_cache(s):
    _plain_append(s, "k")
    _plain_append(s, "v")
    return [_plain_read(s, "k"), _plain_read(s, "v")]


def _dense(s, name):
    """[batch, kv_heads, tokens, dim] values of the cache."""
    slot = s["table"].long()
    x = _values(s[name + "_cache"][slot], s[name + "_scale"][slot])
    b, pages, heads, page, dim = x.shape
    return x.transpose(1, 2).reshape(b, heads, pages * page, dim)[:, :, : s["max_total"]]


def _plain_attention(s):
    b, hq, hk, d, most = s["batch"], s["heads"], s["kv_heads"], s["dim"], s["max_new"]
    tokens = s["q"].shape[0]
    row = (s["cu_new"][:-1, None] + torch.arange(most, device="cuda")[None, :]).clamp(max=tokens - 1)
    q = s["q"][row].float().view(b, most, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    scores = (q @ _dense(s, "k").transpose(2, 3)) * s["softmax_scale"]
    scores = scores.view(b, hq, most, -1)
    place = (s["past"][:, None] + torch.arange(most, device="cuda")[None, :])[:, None, :, None]
    token = torch.arange(s["max_total"], device="cuda")[None, None, None, :]
    seen = token <= place
    if s["window"]:
        seen = seen & (token > place - s["window"])
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(3, keepdim=True)
    weights = scores.sub_(torch.where(top > -math.inf, top, torch.zeros_like(top))).exp_()
    total = weights.sum(3, keepdim=True)
    out = weights.view(b, hk, -1, weights.shape[3]) @ _dense(s, "v")
    out = out.view(b, hq, most, d) / torch.where(total > 0, total, torch.ones_like(total))
    seq, index = _packed(s["cu_new"], tokens)
    return out[seq, :, index].half()


# ------------------------------------------------------------------------------ the library
def _own(s):
    from paper_2608_10103_b200 import binding as lib

    if s["op"] == "rotary":
        return lib.rotary_fp16(s["q"], s["k_new"], s["positions"], s["inv_freq"], s["sections"], pairs=s["pairs"])
    if s["op"] == "prompt":
        return lib.attention_fp16(s["q"], s["k_new"], s["v_new"], s["cu_new"], s["max_new"],
                                  softmax_scale=s["softmax_scale"], causal=s["causal"], window=s["window"])
    cache = (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    if s["op"] == "cache":
        lib.kv_append_u4(cache, s["k_new"], s["v_new"], s["cu_new"], s["past"], s["table"], s["max_new"])
        return lib.kv_read_u4(cache, s["cu_read"], s["first_read"], s["table"], s["max_read"],
                              tokens=s["tokens_read"])
    return lib.kv_attention_u4(s["q"], cache, s["cu_new"], s["total"], s["table"], s["max_new"],
                               softmax_scale=s["softmax_scale"], window=s["window"])


def run(state):
    if own:
        return _own(state)
    return {"rotary": _plain_rotary, "prompt": _plain_prompt, "cache": _plain_cache,
            "attention": _plain_attention}[state["op"]](state)


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotary":
        half, outs = case["rotary"] // 2, []
        which = sum(([a] * n for a, n in enumerate(s["sections"])), [])
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           s["positions"].double()[which].mul(s["inv_freq"].double()[:, None]).t())
        for x in (s["q"], s["k_new"]):
            y = x.double()
            part = y[..., : case["rotary"]]
            z = part.unflatten(2, (2, half)).transpose(2, 3) if case["pairs"] == "halves" else part.unflatten(2, (half, 2))
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
            z = z.transpose(2, 3) if case["pairs"] == "halves" else z
            outs.append(torch.cat((z.reshape(part.shape), y[..., case["rotary"]:]), dim=2))
        return outs
    past, new = _lengths(case)
    if sum(n * (p + n) for p, n in zip(past, new)) * hq * d > 4e12:
        return None

    def attend(q, k, v, first, causal):
        """q [n, hq, d] at positions `first` ..., k and v [hk, tokens, d]."""
        rows, token = [], torch.arange(k.shape[1], device="cuda")
        for lo in range(0, q.shape[0], 256):
            part = q[lo: lo + 256].view(-1, hk, hq // hk, d)
            logits = torch.einsum("thgd,hld->thgl", part, k) * s["softmax_scale"]
            place = first + lo + torch.arange(part.shape[0], device="cuda")
            if causal:
                hidden = token[None, :] > place[:, None]
                if case["window"]:
                    hidden |= token[None, :] <= place[:, None] - case["window"]
                logits.masked_fill_(hidden[:, None, None, :], -math.inf)
            rows.append(torch.einsum("thgl,hld->thgd", logits.softmax(3), v).reshape(-1, hq, d))
        return torch.cat(rows)

    if case["op"] == "prompt":
        parts = zip(*(s[n].double().split(new) for n in ("q", "k_new", "v_new")))
        return torch.cat([attend(q, k.transpose(0, 1), v.transpose(0, 1), 0, case["causal"]) for q, k, v in parts])
    page = case["page"]

    def held(name, i, lo, hi):
        """Values of tokens lo .. hi - 1 of sequence i as they stand in the cache, [tokens, hk, d]."""
        slots = s["table"][i, lo // page: -(-hi // page)].long()
        code, scale = s[name + "_cache"][slots].transpose(1, 2).long(), s[name + "_scale"][slots].transpose(1, 2).double()
        code = torch.cat(((code % 16).unsqueeze(4), (code // 16).unsqueeze(4)), dim=4).flatten(3).double()
        x = torch.addcmul(scale[..., 1:].expand_as(code), code, scale[..., :1].expand_as(code))
        return x.reshape(-1, hk, d)[lo % page: lo % page + hi - lo]

    if case["op"] == "cache":
        outs = []
        for name in ("k", "v"):
            parts, at = [], 0
            for i, (p, n) in enumerate(zip(past, new)):
                x = s[name + "_new"][at: at + n].double()
                at += n
                low = x.amin(2, keepdim=True)
                step = ((x.amax(2, keepdim=True) - low) / 15.0).half().double()  # as it is stored
                code = torch.round((x - low) / torch.where(step > 0, step, torch.ones_like(step))).clamp(0, 15)
                begin = p + n - min(case["read"], p + n)
                if begin < p:
                    parts.append(held(name, i, begin, p))
                parts.append((low + code * step)[max(0, begin - p):])
            outs.append(torch.cat(parts))
        return outs
    out, at = [], 0
    for i, (p, n) in enumerate(zip(past, new)):
        k, v = (held(name, i, 0, p + n).transpose(0, 1) for name in ("k", "v"))
        out.append(attend(s["q"][at: at + n].double(), k, v, p, True))
        at += n
    return torch.cat(out)
