"""Workloads of the operators around the integer and FP16 products: linear layers with their
epilogue, row quantisation in front of an integer product, an INT8 key/value cache (written and
read back) and attention over that cache.

`run` takes one pass through an operator: in elementary torch operations in 32 bits (`own` false)
or through the library's entry points (`own` true), on the same inputs.
"""
import math

import torch

own = False

_DTYPES = {"fp16": torch.float16, "fp32": torch.float32}
_QMAX = {"s8": 127.0, "s4": 7.0}
_ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ---------------------------------------------------------------------------------- cases
def listed():
    return [
        # One token through an output projection: bound by reading the FP16 weights once.
        dict(name="linear_fp16_token", op="linear", m=1, n=4096, k=4096, act="none", bias=True,
             residual=True, out="fp16"),
        # A few hundred rows of odd sizes, every epilogue stage, FP32 result.
        dict(name="linear_fp16_odd", op="linear", m=333, n=1001, k=1096, act="gelu", bias=True,
             residual=True, out="fp32"),
        # The first product of a wide feed-forward block over a long prompt: bound by the tensor cores.
        dict(name="linear_fp16_prompt", op="linear", m=4096, n=16384, k=4096, act="gelu_tanh",
             bias=True, residual=False, out="fp16"),
        # Decoding with a small batch: FP16 activations quantised to INT8, then the INT8 product.
        dict(name="qlinear_s8_decode", op="qlinear", prec="s8", m=8, n=8192, k=8192, act="none",
             bias=False, residual=True, out="fp16"),
        # Decoding with a larger batch on packed 4-bit operands, a wide feed-forward block.
        dict(name="qlinear_s4_decode", op="qlinear", prec="s4", m=32, n=28672, k=8192, act="silu",
             bias=True, residual=False, out="fp16"),
        # A prompt through an INT8 projection back onto the residual stream, row count not a tile multiple.
        dict(name="qlinear_s8_prompt", op="qlinear", prec="s8", m=2000, n=8192, k=8192, act="none",
             bias=True, residual=True, out="fp16"),
        # Each sequence of a batch appends one token; the block it lands in is read back.
        dict(name="cache_token", op="cache", batch=64, heads=32, kv_heads=8, dim=128, page=16,
             past=4096, new=1, read=16),
        # A prompt is written to the cache behind a shared prefix, and everything is read back.
        dict(name="cache_prompt", op="cache", batch=4, heads=32, kv_heads=8, dim=128, page=64,
             past=1000, new=8192, read=9192),
        # One short conversation, one token: latency.
        dict(name="attention_short", op="attention", batch=1, heads=32, kv_heads=8, dim=128, page=16,
             length=1000, new=1, window=0),
        # A batch of conversations of very different lengths, one token each.
        dict(name="attention_batch", op="attention", batch=64, heads=32, kv_heads=8, dim=128, page=16,
             length=8192, new=1, window=0),
        # One document of 128 K tokens, four tokens to verify, every head with its own keys.
        dict(name="attention_long", op="attention", batch=1, heads=16, kv_heads=16, dim=64, page=64,
             length=131071, new=4, window=0),
        # A chunk of a long prompt against what is already cached.
        dict(name="attention_chunk", op="attention", batch=2, heads=32, kv_heads=8, dim=128, page=64,
             length=8192, new=2048, window=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("linear", "qlinear", "cache", "attention"))
        if op in ("linear", "qlinear"):
            c = dict(op=op, m=_log(rng, 1, 4096), n=_log(rng, 64, 28672), k=32 * _log(rng, 2, 512),
                     act=rng.choice(_ACTIVATIONS), bias=rng.random() < 0.6,
                     residual=rng.random() < 0.5, out=rng.choice(("fp16", "fp16", "fp32")))
            if op == "qlinear":
                c["prec"] = rng.choice(("s8", "s4"))
            else:
                c["k"] += rng.choice((0, 8, 16, 24))
        else:
            kv_heads = rng.choice((1, 2, 4, 8, 16))
            c = dict(op=op, batch=_log(rng, 1, 128), heads=kv_heads * rng.choice((1, 2, 3, 4, 8)),
                     kv_heads=kv_heads, dim=rng.choice((64, 128, 256)), page=rng.choice((16, 32, 64, 128)))
            new = 1 if rng.random() < 0.5 else _log(rng, 2, 4096)
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
    return case["m"] * case["n"]


def _spread(most, count, least=0):
    """`count` lengths in [least, most], spread evenly in no particular order, the first the largest."""
    return [most - int((most - least) * ((i * 0.6180339887498949) % 1.0)) for i in range(count)]


def _lengths(case):
    """Per sequence: tokens cached before the call, tokens the call adds (already in the cache for attention)."""
    b = case["batch"]
    new = _spread(case["new"], b, 1 if case["new"] == 1 else max(1, case["new"] // 2))
    if case["op"] == "cache":
        return _spread(case["past"], b), new
    total = [max(t, n) for t, n in zip(_spread(case["length"], b, 1), new)]
    return [t - n for t, n in zip(total, new)], new


def work(case):
    if case["op"] in ("linear", "qlinear"):
        m, n, k = case["m"], case["n"], case["k"]
        weight = {"s8": n * k, "s4": n * k // 2}.get(case.get("prec"), 2 * n * k)
        out = 2 if case["out"] == "fp16" else 4
        by = 2 * m * k + weight + m * n * out * (2 if case["residual"] else 1)
        by += 4 * n if case["bias"] else 0
        by += 4 * n if case["op"] == "qlinear" else 0
        return {"bytes": by, "flops": 2.0 * m * n * k}
    past, new = _lengths(case)
    values = case["kv_heads"] * case["dim"]
    if case["op"] == "cache":
        read = sum(min(case["read"], p + n) for p, n in zip(past, new))
        return {"bytes": 2 * values * (3 * sum(new) + 3 * read), "flops": 0.0}
    pairs = seen = 0
    for p, n in zip(past, new):
        w = case["window"] or (p + n)
        seen += min(p + n, n - 1 + w)
        # query i at position p + i sees min(p + i + 1, w) tokens
        full = max(0, min(n, w - p - 1))
        pairs += full * (p + 1) + full * (full - 1) // 2 + (n - full) * min(w, p + n)
    by = 2 * values * seen + 2 * 2 * sum(new) * case["heads"] * case["dim"]
    return {"bytes": by, "flops": 4.0 * pairs * case["heads"] * case["dim"]}


# --------------------------------------------------------------------------------- inputs
def _pack_s4(q):
    q = q.to(torch.int32) & 15
    return (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = dict(case)
    if case["op"] in ("linear", "qlinear"):
        m, n, k = case["m"], case["n"], case["k"]
        x = normal(m, k)
        x[:, :: max(1, k // 7)] *= 8.0  # a few channels are much larger than the rest, as in trained models
        s["x"] = x.half()
        w = normal(n, k) / math.sqrt(k)
        if case["op"] == "linear":
            s["w"] = w.half()
        else:
            top = _QMAX[case["prec"]]
            s["col_scale"] = w.abs().amax(1) / top
            q = torch.round(w / s["col_scale"][:, None]).clamp(-top, top).to(torch.int8)
            s["w"] = _pack_s4(q) if case["prec"] == "s4" else q
        s["bias"] = normal(n) * 0.5 if case["bias"] else None
        s["residual"] = normal(m, n).to(_DTYPES[case["out"]]) if case["residual"] else None
        s["out_dtype"] = _DTYPES[case["out"]]
        return s
    past, new = _lengths(case)
    b, hk, d, page = case["batch"], case["kv_heads"], case["dim"], case["page"]
    pages = [-(-(p + n) // page) for p, n in zip(past, new)]
    total = sum(pages) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((b, max(pages)), dtype=torch.int32, device="cuda")
    valid = torch.arange(max(pages), device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    table[valid] = order[: sum(pages)]
    s["table"], s["spare"] = table, order[-1].long()
    for name in ("k", "v"):
        s[name + "_cache"] = (normal(total, hk, page, d) * 36.0).round().clamp(-127, 127).to(torch.int8)
        s[name + "_scale"] = 0.02 + 0.02 * torch.rand((total, hk), generator=g, device="cuda")
    # the new tokens' queries, keys and values as one projection leaves them: one row per token
    qkv = normal(sum(new), (case["heads"] + 2 * hk) * d).half()
    hq = case["heads"]
    s["q"] = qkv[:, : hq * d].view(-1, hq, d)
    s["k_new"] = qkv[:, hq * d: (hq + hk) * d].view(-1, hk, d)
    s["v_new"] = qkv[:, (hq + hk) * d:].view(-1, hk, d)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def starts(counts):
        return ints([sum(counts[:i]) for i in range(len(counts) + 1)])

    s["cu_new"], s["past"] = starts(new), ints(past)
    s["total"] = ints([p + n for p, n in zip(past, new)])
    s["max_new"], s["max_total"] = max(new), max(p + n for p, n in zip(past, new))
    if case["op"] == "cache":
        read = [min(case["read"], p + n) for p, n in zip(past, new)]
        s["cu_read"], s["max_read"], s["tokens_read"] = starts(read), max(read), sum(read)
        s["first_read"] = ints([p + n - r for p, n, r in zip(past, new, read)])
    else:
        s["softmax_scale"] = 1.0 / math.sqrt(d)
    return s


# ------------------------------------------------------------------------------- plain form
def _activate(x, name):
    if name == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    return x


def _finish(y, s):
    if s["bias"] is not None:
        y = y + s["bias"].to(y.dtype)
    y = _activate(y, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].to(y.dtype)
    return y


def _unpack_s4(p):
    p = p.to(torch.int32)
    both = torch.stack((p & 15, p >> 4), dim=2).flatten(1)
    return torch.where(both > 7, both - 16, both)


def _plain_linear(s):
    return _finish(s["x"].float() @ s["w"].float().t(), s).to(s["out_dtype"])


def _plain_qlinear(s):
    top = _QMAX[s["prec"]]
    x = s["x"].float()
    amax = x.abs().amax(1)
    most = torch.full_like(amax, top)  # (a tensor: division by a Python number is a product with its inverse)
    scale = amax / most
    inverse = torch.where(amax > 0, most / amax, torch.zeros_like(amax))
    q = torch.round(x * inverse[:, None]).clamp(-top, top)
    w = (_unpack_s4(s["w"]) if s["prec"] == "s4" else s["w"]).float()
    y = (q @ w.t()) * scale[:, None] * s["col_scale"][None, :]
    return [_finish(y, s).to(s["out_dtype"]), scale]


def _packed(cu, tokens):
    """Per row of the packed order: its sequence and its place among that sequence's rows."""
    seq = torch.repeat_interleave(torch.arange(cu.shape[0] - 1, device="cuda"), cu[1:] - cu[:-1],
                                  output_size=tokens)
    return seq, torch.arange(tokens, device="cuda") - cu[seq]


def _plain_append(s, name):
    """The pages that get new tokens, as [batch, pages, heads, page, dim], requantised as a whole."""
    cache, scale, fresh = s[name + "_cache"], s[name + "_scale"], s[name + "_new"].float()
    page = s["page"]
    first = s["past"] // page
    count = (s["max_new"] + page - 2) // page + 1
    ids = first[:, None] + torch.arange(count, device="cuda")[None, :]
    touched = ids * page < s["total"][:, None]
    slot = torch.gather(s["table"], 1, ids.clamp(max=s["table"].shape[1] - 1).long()).long()
    at = ids[:, :, None] * page + torch.arange(page, device="cuda")  # token positions [batch, pages, page]
    is_old = at < s["past"][:, None, None]
    is_new = (at >= s["past"][:, None, None]) & (at < s["total"][:, None, None])
    row = (s["cu_new"][:-1, None, None] + at - s["past"][:, None, None]).clamp(0, fresh.shape[0] - 1).long()
    x = torch.where(is_new[..., None, None], fresh[row], torch.zeros((), device="cuda"))
    x = x.transpose(2, 3)  # [batch, pages, heads, page, dim]
    old = torch.where(is_old[:, :, None, :, None], cache[slot].float(), torch.zeros((), device="cuda"))
    was = torch.where(is_old[:, :, :1], scale[slot], torch.zeros((), device="cuda"))  # [batch, pages, heads]
    now = torch.maximum(was, x.abs().amax((3, 4)) / torch.full_like(was, 127.0))
    inverse = torch.where(now > 0, 1.0 / now, torch.zeros((), device="cuda"))
    codes = torch.round(x * inverse[..., None, None]) + torch.round(old * (was * inverse)[..., None, None])
    codes = codes.clamp(-127, 127).to(torch.int8)
    keep = ~(is_old | is_new)[:, :, None, :, None]
    codes = torch.where(keep, cache[slot], codes)
    slot = torch.where(touched, slot, s["spare"])  # a page that no sequence owns
    cache[slot] = codes
    scale[slot] = now


def _plain_read(s, name):
    seq, place = _packed(s["cu_read"], s["tokens_read"])
    at = s["first_read"][seq] + place
    slot = s["table"][seq, at // s["page"]].long()
    values = s[name + "_cache"][slot, :, at % s["page"]].float()
    return (values * s[name + "_scale"][slot][:, :, None]).half()


def _plain_cache(s):
    _plain_append(s, "k")
    _plain_append(s, "v")
    return [_plain_read(s, "k"), _plain_read(s, "v")]


def _dense(s, name):
    """[batch, kv_heads, tokens, dim] values of the cache."""
    slot = s["table"].long()
    x = s[name + "_cache"][slot].float() * s[name + "_scale"][slot][..., None, None]
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

    if s["op"] == "linear":
        return lib.gemm_fp16_linear(s["x"], s["w"], bias=s["bias"], activation=s["act"],
                                    residual=s["residual"], out_dtype=s["out_dtype"])
    if s["op"] == "qlinear":
        q, scale = lib.gemm_quantize_rows(s["x"], s["prec"])
        product = lib.gemm_s8_linear if s["prec"] == "s8" else lib.gemm_s4_linear
        return [product(q, s["w"], scale, s["col_scale"], bias=s["bias"], activation=s["act"],
                        residual=s["residual"], out_dtype=s["out_dtype"]), scale]
    cache = (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    if s["op"] == "cache":
        lib.kv_append_s8(cache, s["k_new"], s["v_new"], s["cu_new"], s["past"], s["table"], s["max_new"])
        return lib.kv_read_s8(cache, s["cu_read"], s["first_read"], s["table"], s["max_read"],
                              tokens=s["tokens_read"])
    return lib.kv_attention_s8(s["q"], cache, s["cu_new"], s["total"], s["table"], s["max_new"],
                               softmax_scale=s["softmax_scale"], window=s["window"])


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "qlinear": _plain_qlinear, "cache": _plain_cache,
            "attention": _plain_attention}[state["op"]](state)


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("linear", "qlinear"):
        x = s["x"].double()
        if case["op"] == "linear":
            y, scale = x @ s["w"].double().t(), None
        else:
            top = _QMAX[case["prec"]]
            w = s["w"].long()
            if case["prec"] == "s4":
                w = torch.stack((((w & 15) ^ 8) - 8, ((w >> 4) ^ 8) - 8), dim=2).flatten(1)
            scale = x.abs().max(dim=1).values / top
            code = torch.round(x / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None])
            y = (code @ w.double().t()) * torch.outer(scale, s["col_scale"].double())
        if s["bias"] is not None:
            y += s["bias"].double()
        if case["act"] == "relu":
            y = y.clamp(min=0)
        elif case["act"] == "gelu":
            y = y * torch.special.ndtr(y)
        elif case["act"] == "gelu_tanh":
            y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
        elif case["act"] == "silu":
            y = y * torch.sigmoid(y)
        if s["residual"] is not None:
            y += s["residual"].double()
        return y if scale is None else [y, scale]
    page, d, hk = case["page"], case["dim"], case["kv_heads"]
    past, new = _lengths(case)
    if case["op"] == "cache":
        outs = []
        for name in ("k", "v"):
            parts, at = [], 0
            for i, (p, n) in enumerate(zip(past, new)):
                fresh = s[name + "_new"][at: at + n].double()
                at += n
                count = min(case["read"], p + n)
                lo = (p + n - count) // page
                slots = s["table"][i, lo: -(-(p + n) // page)].long()
                scales = s[name + "_scale"][slots].double()
                codes = s[name + "_cache"][slots].double()  # [pages, heads, page, dim]
                values = torch.zeros((len(slots) * page, hk, d), dtype=torch.float64, device="cuda")
                values[: p - lo * page if p > lo * page else 0] = \
                    codes.transpose(1, 2).reshape(-1, hk, d)[: max(0, p - lo * page)]
                is_new = torch.zeros(len(slots) * page, dtype=torch.bool, device="cuda")
                n_read = p + n - max(p, lo * page)
                is_new[max(p, lo * page) - lo * page: p + n - lo * page] = True
                values[is_new] = fresh[n - n_read:]
                values = values.view(-1, page, hk, d)
                is_new = is_new.view(-1, page)
                has_old = (torch.arange(len(slots), device="cuda") + lo) * page < p
                # (whole pages are looked at, so new tokens in front of the first one read count too)
                peak = (values.abs() * is_new[:, :, None, None]).amax((1, 3)) / 127.0
                now = torch.maximum(peak, scales * has_old[:, None])
                step = torch.where(now > 0, now, torch.ones_like(now))[:, None, :, None]
                real = torch.where(is_new[:, :, None, None], values, values * scales[:, None, :, None])
                real = (torch.round(real / step) * step).view(-1, hk, d)
                parts.append(real[p + n - count - lo * page: p + n - lo * page])
            outs.append(torch.cat(parts))
        return outs
    hq, group = case["heads"], case["heads"] // hk
    if sum(n * (p + n) for p, n in zip(past, new)) * hq * d > 4e12:
        return None
    out, at = [], 0
    for i, (p, n) in enumerate(zip(past, new)):
        slots = s["table"][i, : -(-(p + n) // page)].long()
        kv = []
        for name in ("k", "v"):
            x = s[name + "_cache"][slots].double() * s[name + "_scale"][slots].double()[..., None, None]
            kv.append(x.permute(1, 0, 2, 3).reshape(hk, -1, d)[:, : p + n])
        q = s["q"][at: at + n].double()
        at += n
        token = torch.arange(p + n, device="cuda")
        rows = []
        for lo in range(0, n, 256):
            place = p + torch.arange(lo, min(n, lo + 256), device="cuda")
            hidden = token[None, :] > place[:, None]
            if case["window"]:
                hidden |= token[None, :] <= place[:, None] - case["window"]
            part = q[lo: lo + 256].view(-1, hk, group, d)
            logits = torch.einsum("thgd,hld->thgl", part, kv[0]) * s["softmax_scale"]
            logits.masked_fill_(hidden[:, None, None, :], -math.inf)
            rows.append(torch.einsum("thgl,hld->thgd", logits.softmax(3), kv[1]).reshape(-1, hq, d))
        out.append(torch.cat(rows))
    return torch.cat(out)
