"""Performance cases of the key/value cache and its attention: what a program that serves a model calls
between the qkv projection and the output projection of a decoder layer.

    kv_append   rotates queries and keys by their positions and puts keys and values into a paged cache
                (bf16, or MXFP4: E2M1 codes with one E8M0 scale per 32 values)
    kv_read     reads cached rows back as bf16
    attention   causal attention over the paged cache, with an optional sliding window and first tokens that
                stay visible; for prompts, chunks of prompts and single tokens
    shared      the same where all sequences begin with one prefix, whose pages are read once for all

Head counts are those of Llama-3.1-8B (32 query heads, 8 key/value heads of 128), Qwen2.5-7B (28, 4) and
Qwen3-30B-A3B (32, 4), and generic ones.
"""

import math
import random

import numpy as np
import torch

own = False

ROPE_BASE = 10000.0


def _case(name, op, fmt, seqs, new, ctx, hq, hkv, dim, page, window=0, sinks=0, prefix=0, pad=0):
    """new: rows of the longest sequence of the call, ctx: its cached tokens beyond the prefix, the new ones among them;
    the other sequences are shorter.  pad: rows behind the last sequence."""
    c = {"name": name, "op": op, "fmt": fmt, "seqs": seqs, "new": new, "ctx": ctx, "hq": hq, "hkv": hkv, "dim": dim,
         "page": page, "window": window, "sinks": sinks, "prefix": prefix, "pad": pad}
    if not name:
        del c["name"]
    return c


def listed():
    return [
        # one token of one sequence, Llama-3.1-8B heads: the smallest call
        _case("append_b1_bf16", "append", "bf16", 1, 1, 512, 32, 8, 128, 16),
        # a prompt batch behind the qkv linear, Llama-3.1-8B at 2048 rows a prompt, ragged, with padding rows
        _case("append_prefill_bf16", "append", "bf16", 6, 2048, 2048, 32, 8, 128, 64, pad=37),
        # a decode batch of Qwen2.5-7B on an FP4 cache, its rows read back
        _case("append_read_b96_mx", "append", "mx", 96, 1, 700, 28, 4, 128, 32),
        # a long prompt into an FP4 cache, its rows read back (what a prefix export does)
        _case("append_read_prefill_mx", "append", "mx", 3, 8192, 8192, 32, 8, 128, 16),
        # one token of one conversation, Llama-3.1-8B heads: latency counts
        _case("decode_b1_bf16", "attention", "bf16", 1, 1, 8191, 32, 8, 128, 16),
        # a decode batch with a sliding window and sinks, contexts of all lengths
        _case("decode_b64_window_bf16", "attention", "bf16", 64, 1, 6000, 32, 8, 128, 64, window=4096, sinks=4),
        # a decode batch over long contexts on an FP4 cache, Llama-3.1-8B heads
        _case("decode_b24_long_mx", "attention", "mx", 24, 1, 32768, 32, 8, 128, 32),
        # one long prompt, Llama-3.1-8B heads: the largest product
        _case("prefill_8k_bf16", "attention", "bf16", 1, 8192, 8192, 32, 8, 128, 64),
        # prompts with a sliding window and sinks on an FP4 cache, Qwen3-30B-A3B heads, ragged
        _case("prefill_window_mx", "attention", "mx", 3, 4500, 4500, 32, 4, 128, 16, window=1000, sinks=16, pad=9),
        # a chunk of a prompt over what is cached already, heads of 64
        _case("chunk_d64_bf16", "attention", "bf16", 2, 500, 12000, 16, 4, 64, 32),
        # a decode batch behind one system prompt, Llama-3.1-8B heads
        _case("shared_b64_bf16", "shared", "bf16", 64, 1, 400, 32, 8, 128, 64, prefix=8192),
        # a few drafted tokens a sequence behind one prompt on an FP4 cache, Qwen2.5-7B heads
        _case("shared_b40_draft_mx", "shared", "mx", 40, 4, 900, 28, 4, 128, 16, prefix=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "shared"])
    fmt = rng.choice(["bf16", "mx"])
    hq, hkv = rng.choice([(32, 8), (28, 4), (32, 4), (16, 4), (8, 8), (24, 8), (16, 1)])
    dim, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    window, sinks, prefix = 0, 0, 0
    if op == "append":
        new = rng.choice([1, _log(rng, 2, 4096)])
        seqs = max(1, min(_log(rng, 1, 256), 12288 // new))
        ctx = new + rng.randrange(0, 1024)
    else:
        kind = rng.choice(["decode", "few", "chunk", "prompt"]) if op == "attention" else rng.choice(["decode", "few"])
        if kind == "prompt":
            new = ctx = _log(rng, 16, 6000)
        else:
            new = {"decode": 1, "few": rng.randrange(2, 12), "chunk": _log(rng, 12, 700)}[kind]
            ctx = new + _log(rng, 1, 16000 if op == "attention" else 1500)
        if op == "shared":
            prefix = page * max(1, _log(rng, 256, 12000) // page)
        elif rng.random() < 0.5:
            window, sinks = _log(rng, 16, 4096), rng.choice([0, 1, 4, 64])
        whole = prefix + ctx
        # the plain form's scores, and its keys, stay below those of the largest listed cases
        most = min(8192 * 8192 * 32 // (new * whole * hq), 24 * 32768 * 8 // (whole * hkv))
        seqs = max(1, min(_log(rng, 1, 96), most))
    return _case("", op, fmt, seqs, new, ctx, hq, hkv, dim, page, window, sinks, prefix, rng.choice([0, 0, rng.randrange(1, 40)]))


def _lengths(case):
    """(rows of every sequence in the call, cached tokens of every sequence with the prefix); the first is the longest."""
    r = random.Random(17 * case["seqs"] + 31 * case["new"] + case["ctx"])
    new, ctx, seqs = case["new"], case["ctx"], case["seqs"]
    rows = [new] + [r.randint(max(1, new // 3), new) for _ in range(seqs - 1)]
    lens = [ctx] + [max(n, r.randint(max(1, ctx // 3), ctx)) for n in rows[1:]]
    if ctx == new:
        lens = list(rows)
    return rows, [n + case["prefix"] for n in lens]


def _visible(case):
    """(pairs of a row and a token it sees, tokens that some row of their sequence sees, the prefix's counted once)."""
    rows, lens = _lengths(case)
    w, s, pre = case["window"] or 1 << 40, case["sinks"], case["prefix"]
    pairs, tokens, shared = 0, 0, 0
    for n, length in zip(rows, lens):
        p = np.arange(length - n, length, dtype=np.int64)
        low = np.maximum(p - w + 1, 0)
        pairs += int((p + 1 - low + np.minimum(low, s)).sum())
        seen = np.zeros(length, dtype=bool)
        seen[:s] = True
        seen[int(low[0]):] = True
        shared = max(shared, int(seen[:pre].sum()))
        tokens += int(seen[pre:].sum())
    return pairs, tokens + shared


def work(case):
    rows, _ = _lengths(case)
    total, hq, hkv, dim = sum(rows), case["hq"], case["hkv"], case["dim"]
    held = 2.0 if case["fmt"] == "bf16" else 0.5 + 1.0 / 32
    if case["op"] == "append":
        b = total * dim * (2.0 * hq * 2 + 2 * hkv * (2.0 + held)) + total * dim * 4.0
        if case["fmt"] == "mx":
            b += total * 2 * hkv * dim * (held + 2.0)   # read back
        return {"bytes": b, "flops": total * dim * 3.0 * (hq + hkv)}
    pairs, tokens = _visible(case)
    return {"bytes": total * hq * dim * 4.0 + 2.0 * tokens * hkv * dim * held, "flops": 4.0 * dim * hq * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

_MAGNITUDE = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_codes(x):
    """x [..., n], n a multiple of 32 -> E2M1 codes [..., n] and E8M0 codes [..., n / 32]: the exponent is
    floor(log2 of the block's largest magnitude) - 2, values round to the nearest, ties to the even code."""
    blocks = x.unflatten(-1, (-1, 32))
    peak = blocks.abs().amax(-1)
    e = torch.where(peak > 0, torch.frexp(peak).exponent - 3, -127).clamp(-127, 127)
    a = torch.ldexp(blocks.abs(), -e.unsqueeze(-1))
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    return (code + 8 * torch.signbit(blocks).to(torch.uint8)).flatten(-2), (e + 127).to(torch.uint8)


def _mx_values(codes, scales, e2m1):
    """E2M1 codes [..., n] and E8M0 codes [..., n / 32] -> fp32 values; e2m1: the 16 codes' values."""
    v = e2m1[codes.to(torch.int32)].unflatten(-1, (-1, 32))
    return torch.ldexp(v, (scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    hq, hkv, dim, page, pre = case["hq"], case["hkv"], case["dim"], case["page"], case["prefix"]
    rows, lens = _lengths(case)
    seqs, total = case["seqs"], sum(rows)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32) * scale

    # every sequence's pages, in no order, as a cache that has served for a while hands them out
    pre_pages = pre // page
    need = [-(-(n - pre) // page) for n in lens]
    pages = pre_pages + sum(need) + 3
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((seqs, pre_pages + max(need)), -1, dtype=torch.int32)
    at = pre_pages
    for s, n in enumerate(need):
        table[s, :pre_pages] = ids[:pre_pages]
        table[s, pre_pages:pre_pages + n] = ids[at:at + n]
        at += n
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32)
    st = {"case": case, "rows": total + case["pad"], "max_rows": max(rows), "max_len": max(lens),
          "offsets": offsets.to(dev), "lens": torch.tensor(lens, dtype=torch.int32).to(dev), "table": table.to(dev),
          "prefix_table": ids[:pre_pages].to(dev), "scale": 1.0 / math.sqrt(dim), "keep": {},
          "e2m1": torch.tensor(_MAGNITUDE + tuple(-m for m in _MAGNITUDE), dtype=torch.float32).to(dev)}

    # the cache: keys with a few strong channels, values with a mean, as projections give them
    shape = (pages, hkv, page, dim)
    if case["fmt"] == "bf16":
        st["k"] = torch.empty(shape, dtype=torch.bfloat16, device=dev)
        st["v"] = torch.empty(shape, dtype=torch.bfloat16, device=dev)
    else:
        for n in ("k", "v"):
            st[n] = torch.zeros(shape[:3] + (dim // 2,), dtype=torch.uint8, device=dev)
            st[n + "_scale"] = torch.zeros(shape[:3] + (dim // 32,), dtype=torch.uint8, device=dev)
    strong = 1.0 + 2.0 * (torch.rand((hkv, 1, dim), generator=g, device=dev) < 0.04)
    mean = normal(hkv, 1, dim, scale=0.5)
    if case["op"] == "append":
        st["cos"], st["sin"] = _tables(max(lens) + 5, dim)
        st["qkv"] = normal(st["rows"], (hq + 2 * hkv) * dim).to(torch.bfloat16)
        st["q_out"] = torch.zeros((st["rows"], hq * dim), dtype=torch.bfloat16, device=dev)
        if case["fmt"] == "bf16":
            st["k"].zero_()
            st["v"].zero_()
        else:
            st["k_rows"] = torch.zeros((st["rows"], hkv * dim), dtype=torch.bfloat16, device=dev)
            st["v_rows"] = torch.zeros((st["rows"], hkv * dim), dtype=torch.bfloat16, device=dev)
        return st
    step = max(1, (1 << 27) // (hkv * page * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        for name, x in (("k", normal(n, hkv, page, dim) * strong), ("v", normal(n, hkv, page, dim) + mean)):
            if case["fmt"] == "bf16":
                st[name][p:p + n] = x
            else:
                c, e = _mx_codes(x)
                st[name][p:p + n] = c[..., 0::2] | (c[..., 1::2] << 4)
                st[name + "_scale"][p:p + n] = e
    st["q"] = normal(st["rows"], hq * dim, scale=1.2).to(torch.bfloat16)
    st["out"] = torch.zeros((st["rows"], hq * dim), dtype=torch.bfloat16, device=dev)
    return st


def _tables(positions, dim):
    """cos and sin [positions, dim / 2] of the rotation, fp32 from angles in 64 bits."""
    j = torch.arange(dim // 2, dtype=torch.float64, device="cuda")
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-2.0 * j / dim)
    return angle.cos().to(torch.float32), angle.sin().to(torch.float32)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    from paper_2606_26587_amd import sharq as S
    case, keep = st["case"], st["keep"]
    if not keep:   # the handles that a program makes once
        keep["cache"] = S.KVCache(case["fmt"], st["k"], st["v"], st.get("k_scale"), st.get("v_scale"))
        keep["batch"] = S.KVBatch(st["offsets"], st["lens"], st["table"], st["rows"], st["max_rows"], st["max_len"])
        if case["op"] != "append":
            keep["prefix"] = st["prefix_table"] if case["prefix"] else None
            size = S.attention_workspace_bytes(keep["cache"], keep["batch"], case["hq"], window=case["window"],
                                               sinks=case["sinks"], prefix_len=case["prefix"])
            keep["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    cache, batch = keep["cache"], keep["batch"]
    if case["op"] == "append":
        nq, nk = case["hq"] * case["dim"], case["hkv"] * case["dim"]
        x = st["qkv"]
        q = S.sharq_kv_append(x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:], cache, batch, cos=st["cos"], sin=st["sin"],
                              q_out=st["q_out"])
        if case["fmt"] == "bf16":
            return {"q": q, "k": st["k"], "v": st["v"]}
        k, v = S.sharq_kv_read(cache, batch, k_out=st["k_rows"], v_out=st["v_rows"])
        return {"q": q, "k": k, "v": v}
    return S.sharq_attention(st["q"], cache, batch, scale=st["scale"], window=case["window"], sinks=case["sinks"],
                             prefix_table=keep["prefix"], prefix_len=case["prefix"], out=st["out"],
                             workspace=keep["ws"])


def _plain(st):
    return _plain_append(st) if st["case"]["op"] == "append" else _plain_attention(st)


def _plain_append(st):
    case = st["case"]
    hq, hkv, dim, page = case["hq"], case["hkv"], case["dim"], case["page"]
    offsets, lens, x = st["offsets"], st["lens"], st["qkv"].float()
    row = torch.arange(st["rows"], device=x.device)
    seq = torch.searchsorted(offsets[1:].contiguous(), row, right=True, out_int32=True)
    live = seq < lens.numel()
    seq = seq.clamp(max=lens.numel() - 1)
    pos = torch.where(live, lens[seq] - offsets[seq + 1] + row, 0)
    c, s = st["cos"][pos][:, None], st["sin"][pos][:, None]

    def turned(y):
        a, b = y[..., :dim // 2], y[..., dim // 2:]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    q = turned(x[:, :hq * dim].unflatten(-1, (hq, dim)))
    k = turned(x[:, hq * dim:(hq + hkv) * dim].unflatten(-1, (hkv, dim)))
    v = x[:, (hq + hkv) * dim:].unflatten(-1, (hkv, dim))
    q = torch.where(live[:, None], q.flatten(1).to(torch.bfloat16), st["q_out"])
    if case["fmt"] == "mx":
        k, v = (torch.where(live[:, None], _mx_values(*_mx_codes(y), st["e2m1"]).flatten(1).to(torch.bfloat16), old)
                for y, old in ((k, st["k_rows"]), (v, st["v_rows"])))
        return {"q": q, "k": k, "v": v}
    n = int(sum(_lengths(case)[0]))
    at = (st["table"][seq, pos // page], pos % page)
    at = (at[0][:n].long(), slice(None), at[1][:n].long())
    st["k"][at] = k[:n].to(torch.bfloat16)
    st["v"][at] = v[:n].to(torch.bfloat16)
    return {"q": q, "k": st["k"], "v": st["v"]}


def _cached(st, name, pages):
    """Cached values of a table of pages [..., n], fp32 [..., hkv, n * page, dim]."""
    pages = pages.clamp(min=0).long()
    x = st[name][pages]
    x = x.float() if st["case"]["fmt"] == "bf16" else _mx_values(_unpack(x), st[name + "_scale"][pages], st["e2m1"])
    return x.movedim(-4, -3).flatten(-3, -2)


def _plain_attention(st):
    case = st["case"]
    hq, hkv, dim, w, sinks = case["hq"], case["hkv"], case["dim"], case["window"], case["sinks"]
    group, seqs, most = hq // hkv, case["seqs"], st["max_rows"]
    offsets, lens = st["offsets"], st["lens"]
    length = st["table"].shape[1] * case["page"]
    k, v = _cached(st, "k", st["table"]), _cached(st, "v", st["table"])
    i = torch.arange(most, device=k.device)
    n = offsets[1:] - offsets[:-1]
    row = (offsets[:-1, None] + i).clamp(max=st["rows"] - 1).long()
    q = st["q"].float()[row].unflatten(-1, (hkv, group, dim))
    q = q.permute(0, 2, 1, 3, 4).reshape(seqs, hkv, most * group, dim)
    pos = (lens - n)[:, None] + i
    t = torch.arange(length, device=k.device)
    seen = t <= pos[..., None]
    if w:
        seen = seen & ((pos[..., None] - t < w) | (t < sinks))
    seen = seen.repeat_interleave(group, 1)[:, None]
    score = torch.matmul(q, k.transpose(-1, -2)).mul_(st["scale"]).masked_fill_(~seen, -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = score.sum(-1, keepdim=True)
    # a token that no row sees may hold anything
    v = torch.where(seen.any(2)[..., None], v, 0)
    o = torch.matmul(score, v) / torch.where(total > 0, total, 1)
    o = o.view(seqs, hkv, most, group, dim).permute(0, 2, 1, 3, 4).reshape(seqs, most, hq * dim)
    live = i < n[:, None]
    out = st["out"].clone()
    out[row[live]] = o[live].to(torch.bfloat16)
    return out


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    rows, lens = _lengths(case)
    hq, hkv, dim, page, group = case["hq"], case["hkv"], case["dim"], case["page"], case["hq"] // case["hkv"]
    half = dim // 2
    start = 0
    if case["op"] == "append":
        q = torch.zeros((st["rows"], hq * dim), dtype=torch.float64, device="cuda")
        kv = {n: (torch.zeros(st[n].shape, dtype=torch.float64, device="cuda") if case["fmt"] == "bf16" else
                  torch.zeros((st["rows"], hkv * dim), dtype=torch.float64, device="cuda")) for n in ("k", "v")}
        for s, (n, length) in enumerate(zip(rows, lens)):
            at = slice(start, start + n)
            start += n
            pos = torch.arange(length - n, length, device="cuda")
            unit = torch.complex(st["cos"][pos].double(), st["sin"][pos].double())[:, None]
            x = st["qkv"][at].double().view(n, hq + 2 * hkv, dim)
            z = torch.complex(x[:, :hq + hkv, :half], x[:, :hq + hkv, half:]) * unit
            x[:, :hq + hkv] = torch.cat((z.real, z.imag), -1)
            q[at] = x[:, :hq].reshape(n, -1)
            for name, y in (("k", x[:, hq:hq + hkv]), ("v", x[:, hq + hkv:])):
                if case["fmt"] == "bf16":
                    kv[name][st["table"][s][pos // page].long(), :, pos % page] = y
                else:
                    kv[name][at] = _nearest(y.reshape(n, -1, 32)).reshape(n, -1)
        return {"q": q, **kv}
    out = torch.zeros((st["rows"], hq * dim), dtype=torch.float64, device="cuda")
    for s, (n, length) in enumerate(zip(rows, lens)):
        at = slice(start, start + n)
        start += n
        ids = st["table"][s][:-(-length // page)].long()
        t = torch.arange(length, device="cuda")
        p = torch.arange(length - n, length, device="cuda")[:, None]
        hidden = t > p
        if case["window"]:
            hidden |= (t <= p - case["window"]) & (t >= case["sinks"])
        q = st["q"][at].double().view(n, hq, dim)
        for h in range(hkv):
            k, v = (_held(st, name, ids, h)[:length] for name in ("k", "v"))
            for m in range(group):
                z = q[:, h * group + m] @ k.T * st["scale"]
                z[hidden] = -math.inf
                out[at, (h * group + m) * dim:(h * group + m + 1) * dim] = torch.softmax(z, -1) @ v
    return out


def _nearest(x):
    """Blocks of 32 values [..., 32] in 64 bits -> the MXFP4 values that they are held as."""
    peak = x.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.floor(torch.log2(peak.clamp(min=2.0 ** -125))) - 2)
    a = (x / unit).abs().clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step * unit, x)


def _held(st, name, ids, h):
    """One head's cached values of a row of pages, in 64 bits [tokens, dim]."""
    x = st[name][ids, h].flatten(0, 1)
    if st["case"]["fmt"] == "bf16":
        return x.double()
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    c = torch.stack((x % 16, x // 16), -1).flatten(1).long()
    v = grid[c % 8] * (1 - 2 * (c // 8)).double()
    e = st[name + "_scale"][ids, h].flatten(0, 1).double() - 127
    return v * torch.exp2(e).repeat_interleave(32, 1)
