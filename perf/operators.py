"""The operators between pruning and the answer, as cases that can be prepared, run and compared.

A case is a dict of plain values.  `op` says which entry point it goes through:

  tables  binding.map_pages: block tables, slots and positions of a ragged batch, from lengths on the device
  rope    binding.qk_norm_rope: norms of queries and keys per head and the rotation by position, in one pass
  write   binding.cache_write: keys and values into pages of 8-bit codes with a scale per page and head
  attend  binding.cache_attend: attention of ragged queries over those pages

Lengths are what pruning leaves of page images (337 of 400 tokens and the like); rows behind the last sequence are
there because a run with a dynamic ratio fills its output only in part.  Heads are 10 of 128 (the width of 1280 that
the library prunes at), or generic grouped ones.  `own` chooses the library's operators over their plain form.

The scale of a block is the smallest power of two that takes its largest value to at most 127, so codes and scales
are exact and are returned as they are held: they have to be equal.
"""
import math

import numpy as np
import torch

own = False

GOLDEN = 0.6180339887498949
EPS = 1e-6


def _tables(name, batch, new_lo, new_hi, ctx_lo, ctx_hi, page, pad, index):
    return {"name": name, "op": "tables", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "page": page, "pad": pad, "index": index}


def _rope(name, rows, q_heads, kv_heads, dim, rotary, interleaved, norm, far, dtype, pad):
    return {"name": name, "op": "rope", "rows": rows, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary,
            "interleaved": interleaved, "norm": norm, "far": far, "dtype": dtype, "pad": pad}


def _write(name, batch, new_lo, new_hi, ctx_lo, ctx_hi, kv_heads, dim, page, dtype, pad):
    return {"name": name, "op": "write", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "pad": pad}


def _attend(name, batch, new_lo, new_hi, ctx_lo, ctx_hi, q_heads, kv_heads, dim, page, causal=True):
    return {"name": name, "op": "attend", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "page": page, "causal": causal}


def listed():
    return [
        # one decode step of a serving batch: 64 requests get a token each, a page where the last is full
        _tables("tables 64 steps", 64, 1, 1, 200, 1500, 64, 0, False),
        # the pruned batch of a corpus: 1024 images, 300 to 400 tokens left of each, positions from the kept indices
        _tables("tables 1024x300-400", 1024, 300, 400, 0, 40, 64, 30000, True),
        # one decode step: queries and keys of 64 requests, norms and rotation
        _rope("rope 64 steps", 64, 10, 10, 128, 128, False, True, 4000, "bf16", 0),
        # prefill of 64 pruned pages of the large resolution mode, out of a fused projection's rows
        _rope("rope 64x337", 64 * 337, 10, 10, 128, 128, False, True, 450, "bf16", 64 * 63),
        # fp32 storage, grouped heads, half of each head rotated in adjacent pairs, far positions
        _rope("rope fp32 4999 grouped", 4999, 32, 8, 128, 64, True, True, 120000, "fp32", 0),
        # one decode step: a token appended to each of 64 requests' last pages
        _write("write 64 steps", 64, 1, 1, 200, 1500, 10, 128, 64, "bf16", 0),
        # prefill of 64 pruned pages behind a short text prefix
        _write("write 64x300-375", 64, 300, 375, 0, 40, 10, 128, 64, "bf16", 64 * 63),
        # one interactive request: a single token against one page image and its answer so far
        _attend("attend 1x1 of 500", 1, 1, 1, 499, 499, 10, 10, 128, 64),
        # a decode step of a serving batch of pages, lengths mixed
        _attend("attend 64x1 of 350-1500", 64, 1, 1, 349, 1499, 10, 10, 128, 64),
        # a decode step over long documents, grouped heads
        _attend("attend 16x1 of 8k-32k", 16, 1, 1, 8000, 32000, 32, 8, 128, 64),
        # prefill of 64 pruned pages behind a short text prefix
        _attend("attend 64x300-375", 64, 300, 375, 0, 40, 10, 10, 128, 64),
        # prefill of pages with large visual token sets: 2783 tokens kept of 4512
        _attend("attend 8x2783", 8, 2783, 2783, 17, 17, 10, 10, 128, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(10, 10), (32, 8), (16, 2), (12, 4), (7, 7), (8, 1), (5, 1)]


def draw(rng):
    op = rng.choice(["tables", "rope", "write"] + ["attend"] * 3)
    page = rng.choice([16, 32, 64, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    q_heads, kv_heads = rng.choice(HEADS)
    dim = rng.choice([128, 128, 64])
    if op == "tables":
        batch = _log_int(rng, 1, 1024)
        new_hi = _log_int(rng, 1, 400)
        ctx_hi = rng.choice([0, _log_int(rng, 1, 4000)])
        c = _tables("", batch, rng.randint(0 if batch > 1 else 1, new_hi), new_hi, rng.randint(0, ctx_hi), ctx_hi, page,
                    rng.randint(0, 300), rng.random() < 0.5)
    elif op == "rope":
        dim = rng.choice([128, 128, 64, 96, 256])
        rotary = rng.choice([dim, dim, dim // 2, 32])
        rows = _log_int(rng, 1, min(25600, 32_000_000 // ((q_heads + kv_heads) * dim)))
        c = _rope("", rows, q_heads, kv_heads, dim, rotary, rng.random() < 0.3, rng.random() < 0.8, _log_int(rng, 64, 1_000_000),
                  dtype, rng.randint(0, 40))
    elif op == "write":
        batch = _log_int(rng, 1, 256)
        new_hi = _log_int(rng, 1, max(1, min(3000, 27_000_000 // (batch * kv_heads * dim))))
        ctx_hi = rng.choice([0, _log_int(rng, 1, 1500)])
        c = _write("", batch, rng.randint(1, new_hi), new_hi, rng.randint(0, ctx_hi), ctx_hi, kv_heads, dim, page, dtype,
                   rng.randint(0, 100))
    else:
        batch = _log_int(rng, 1, 96)
        family = rng.choice(["step", "step", "few", "prefill", "prefill"])
        if family == "step":
            new_lo = new_hi = 1
        elif family == "few":
            new_hi = rng.randint(2, 12)
            new_lo = rng.randint(1, new_hi)
        else:
            new_hi = _log_int(rng, 13, 2783)
            new_lo = rng.randint(1, new_hi)
        # bounded by the largest listed pass: cached elements, and query-token pairs
        most = min(32000, 536_000_000 // (batch * kv_heads * dim * 2), 600_000_000 // (batch * q_heads * new_hi))
        while most < new_hi + 1:
            batch = max(1, batch // 2)
            new_hi = new_hi if batch > 1 else max(1, new_hi // 2)
            new_lo = min(new_lo, new_hi)
            most = min(32000, 536_000_000 // (batch * kv_heads * dim * 2), 600_000_000 // (batch * q_heads * new_hi))
        ctx_hi = rng.choice([0, 1, 1]) * _log_int(rng, 1, max(1, most - new_hi))
        ctx_lo = rng.randint(0, ctx_hi)
        c = _attend("", batch, new_lo, new_hi, ctx_lo, ctx_hi, q_heads, kv_heads, dim, page, family != "prefill" or rng.random() < 0.8)
    del c["name"]
    return c


def _spread(lo, hi, n, start):
    return [lo + int(((i + start) * GOLDEN % 1.0) * (hi - lo + 1)) for i in range(n)]


def _lengths(case):
    """New tokens of each request and tokens that it has cached before: spread evenly over their ranges, in mixed order."""
    return _spread(case["new_lo"], case["new_hi"], case["batch"], 1), _spread(case["ctx_lo"], case["ctx_hi"], case["batch"], 3)


def _ceil(a, b):
    return -(-a // b)


def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _int(values, dev):
    return torch.tensor(values, dtype=torch.int32, device=dev)


def _batch(case, gen, dev):
    """Offsets, contexts, and a table of pages in shuffled order for a batch that has its pages already."""
    new, ctx = _lengths(case)
    ps = case["page"]
    pages = [_ceil(c + n, ps) for c, n in zip(ctx, new)]
    most = max(max(pages), 1)
    order = torch.randperm(sum(pages) + 1, generator=gen, device=dev).to(torch.int32)
    table = torch.full((case["batch"], most), -1, dtype=torch.int32, device=dev)
    first = np.concatenate([[0], np.cumsum(pages)])
    inside = torch.arange(most, device=dev)[None, :] < _int(pages, dev)[:, None]
    at = _int(first[:-1].tolist(), dev)[:, None] + torch.arange(most, device=dev)[None, :]
    table = torch.where(inside, order[at.clamp(max=sum(pages)).long()], table)
    offsets = _int(np.concatenate([[0], np.cumsum(new)]).tolist(), dev)
    return new, ctx, table, offsets, sum(pages) + 1


def _cache(case, pages, gen, dev):
    """Codes and scales of a filled cache, in the library's layout: keys and values about as large as normed ones are."""
    h, ps, d = case["kv_heads"], case["page"], case["dim"]
    shape = (pages, h, ps, d)
    k = torch.empty(shape, dtype=torch.int8, device=dev)
    v = torch.empty(shape, dtype=torch.int8, device=dev)
    for c in (k, v):
        flat = c.view(-1)
        for lo in range(0, flat.numel(), 1 << 26):
            part = flat[lo:lo + (1 << 26)]
            part.copy_((torch.randn(part.numel(), generator=gen, device=dev) * 36).round().clamp(-127, 127))
    power = torch.randint(-6, -3, (2, pages, h), generator=gen, device=dev).float()
    return k, v, torch.exp2(power[0]), torch.exp2(power[1])


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    op = case["op"]
    if op == "tables":
        new, ctx = _lengths(case)
        ps, rows = case["page"], sum(new) + case["pad"]
        has = [_ceil(c, ps) for c in ctx]
        need = [_ceil(c + n, ps) - a for c, n, a in zip(ctx, new, has)]
        ids = torch.randperm(sum(has) + sum(need) + 9, generator=gen, device=dev).to(torch.int32)
        most = max(max(a + b for a, b in zip(has, need)), 1)
        table = torch.full((case["batch"], most), -1, dtype=torch.int32, device=dev)
        inside = torch.arange(most, device=dev)[None, :] < _int(has, dev)[:, None]
        at = _int(np.concatenate([[0], np.cumsum(has)])[:-1].tolist(), dev)[:, None] + torch.arange(most, device=dev)[None, :]
        table = torch.where(inside, ids[at.clamp(max=ids.numel() - 1).long()], table)
        index = torch.randint(0, 4512, (max(rows, 1),), generator=gen, device=dev, dtype=torch.int32) if case["index"] else None
        return {"case": case, "offsets": _int(np.concatenate([[0], np.cumsum(new)]).tolist(), dev), "ctx": _int(ctx, dev),
                "free": ids[sum(has):].contiguous(), "head": _int([3], dev), "table": table, "index": index, "rows": rows,
                "base": _int(_spread(0, 50, case["batch"], 2), dev) if case["index"] else None,
                "out": tuple(torch.zeros(n, dtype=torch.int32, device=dev) for n in (rows, rows, case["batch"], 2))}
    dtype = torch.float32 if case.get("dtype") == "fp32" else torch.bfloat16
    if op == "rope":
        rows, qh, kh, d = case["rows"] + case["pad"], case["q_heads"], case["kv_heads"], case["dim"]
        x = torch.randn(rows, (qh + 2 * kh) * d, generator=gen, device=dev)
        x *= torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=dev))
        x = x.to(dtype)                                          # a fused projection's rows: queries, keys, values
        pos = torch.randint(0, case["far"], (rows,), generator=gen, device=dev, dtype=torch.int32)
        pos[case["rows"]:] = -1
        s = {"case": case, "q": x[:, :qh * d].view(rows, qh, d), "k": x[:, qh * d:(qh + kh) * d].view(rows, kh, d), "pos": pos,
             "freq": 10000.0 ** (torch.arange(0, case["rotary"], 2, dtype=torch.float64, device=dev) / -case["rotary"]), "wq": None, "wk": None,
             "q_out": torch.zeros(rows, qh, d, dtype=dtype, device=dev), "k_out": torch.zeros(rows, kh, d, dtype=dtype, device=dev)}
        if case["norm"]:
            s["wq"] = (1 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(dtype)
            s["wk"] = (1 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(dtype)
        return s
    new, ctx, table, offsets, pages = _batch(case, gen, dev)
    cache = _cache(case, pages, gen, dev)
    h, d, ps = case["kv_heads"], case["dim"], case["page"]
    if op == "write":
        rows = sum(new) + case["pad"]
        x = torch.randn(rows, 2 * h * d, generator=gen, device=dev)
        x *= torch.exp(0.7 * torch.randn(rows, 1, generator=gen, device=dev))
        x = x.to(dtype)                                          # keys and values beside each other in a row
        req = torch.repeat_interleave(torch.arange(case["batch"], device=dev), _int(new, dev), output_size=sum(new))
        at = _int(ctx, dev)[req] + torch.arange(sum(new), device=dev) - offsets[req]
        slots = torch.full((rows,), -1, dtype=torch.int32, device=dev)
        slots[:sum(new)] = (table[req, at // ps] * ps + at % ps).to(torch.int32)
        return {"case": case, "k": x[:, :h * d].view(rows, h, d), "v": x[:, h * d:].view(rows, h, d), "slots": slots, "cache": cache}
    rows = sum(new)
    q = torch.randn(rows, case["q_heads"], d, generator=gen, device=dev)
    q *= torch.exp(0.5 * torch.randn(1, case["q_heads"], 1, generator=gen, device=dev))      # heads that attend widely, and sharply
    return {"case": case, "q": q.to(torch.bfloat16), "cache": cache, "offsets": offsets, "table": table,
            "lens": _int([a + b for a, b in zip(ctx, new)], dev), "max_q": max(new), "max_len": max(a + b for a, b in zip(ctx, new)),
            "out": torch.zeros(rows, case["q_heads"], d, dtype=torch.bfloat16, device=dev),
            "lse": torch.zeros(rows, case["q_heads"], device=dev)}


def run(state):
    return {"tables": _run_tables, "rope": _run_rope, "write": _run_write, "attend": _run_attend}[state["case"]["op"]](state)


def _run_tables(s):
    if own:
        from paper_2605_00392_b200 import binding
        binding.map_pages(s["offsets"], s["table"], s["free"], s["head"], s["out"], page_size=s["case"]["page"], context_lens=s["ctx"],
                          token_index=s["index"], position_base=s["base"])
        return (s["table"],) + s["out"]
    ps, off, ctx, table = s["case"]["page"], s["offsets"], s["ctx"], s["table"]
    n = off[1:] - off[:-1]
    has = (ctx + ps - 1) // ps
    need = (ctx + n + ps - 1) // ps - has
    start = s["head"] + torch.cumsum(need, 0) - need
    row = torch.arange(s["rows"], device=off.device)
    req = torch.searchsorted(off[1:].contiguous(), row.to(torch.int32), right=True).clamp(max=ctx.numel() - 1)
    real = row < off[-1]
    x = torch.where(real, ctx[req] + row - off[req], 0)
    p = x // ps
    held = table[req, p.clamp(max=table.shape[1] - 1)]
    page = torch.where(p < has[req], held, s["free"][(start[req] + p - has[req]).clamp(0, s["free"].numel() - 1)])
    slots = torch.where(real, page * ps + x % ps, -1).to(torch.int32)
    wide = torch.cat([table, table[:, :1]], 1)                   # rows of no sequence go to a column of their own
    wide[req, torch.where(real, p, table.shape[1])] = page
    pos = s["base"][req] + s["index"] if s["index"] is not None else x
    pos = torch.where(real, pos, -1).to(torch.int32)
    state = torch.cat([s["head"] + need.sum(), torch.zeros_like(s["head"])]).to(torch.int32)
    return wide[:, :-1].contiguous(), slots, pos, (ctx + n).to(torch.int32), state


def _turned(x, w, cos, sin, rotary, interleaved):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    r = y[..., :rotary]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        t = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :rotary // 2], r[..., rotary // 2:]
        t = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([t, y[..., rotary:]], -1)


def _run_rope(s):
    c = s["case"]
    if own:
        from paper_2605_00392_b200 import binding
        binding.qk_norm_rope(s["q"], s["k"], s["pos"], s["freq"], s["wq"], s["wk"], EPS, interleaved=c["interleaved"],
                             q_out=s["q_out"], k_out=s["k_out"])
        return s["q_out"], s["k_out"]
    angle = s["pos"].double()[:, None] * s["freq"][None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    real = (s["pos"] >= 0)[:, None, None]
    return tuple(torch.where(real, _turned(s[n], s[w], cos, sin, c["rotary"], c["interleaved"]).to(s[n].dtype), s[o])
                 for n, w, o in (("q", "wq", "q_out"), ("k", "wk", "k_out")))


def _written(x, slots, codes, scale, ps):
    """Codes and scales after the rows of x have gone to their slots."""
    pages, h = scale.shape
    real = slots >= 0
    page = torch.where(real, slots // ps, pages).long()           # rows of no sequence go to a page of their own
    y = x.float()
    top = torch.zeros(pages + 1, h, device=y.device).scatter_reduce_(0, page[:, None].expand(-1, h), y.abs().amax(-1), "amax")[:-1]
    first = torch.full((pages + 1,), ps, dtype=torch.int32, device=y.device)
    first = first.scatter_reduce_(0, page, (slots % ps).to(torch.int32), "amin")[:-1]
    m, e = torch.frexp(top)                                       # top = m 2^e, 0.5 <= m < 1: 127 2^(e - 7) >= top where m <= 127/128
    want = torch.where(top > 0, torch.ldexp(torch.ones_like(top), e - 7 + (m > 127 / 128).int()), 0)
    old = torch.where((first > 0)[:, None], scale, 0)
    new = torch.where((first < ps)[:, None], torch.maximum(want, old), scale)
    shrink = torch.where(new > 0, scale / new, 1).clamp(max=1)[:, :, None, None]
    earlier = torch.arange(ps, device=y.device) < first[:, None]      # tokens that the page held before
    codes = torch.where((new != scale)[:, :, None, None] & earlier[:, None, :, None], (codes.float() * shrink).round(), codes.float())
    codes = torch.cat([codes, codes[:1]])
    s = torch.cat([new, new[:1]])[page][..., None]
    codes[page, :, torch.where(real, slots % ps, 0).long()] = torch.where(s > 0, y / s, 0).round().clamp(-127, 127)
    return codes[:-1].to(torch.int8), new


def _run_write(s):
    if own:
        from paper_2605_00392_b200 import binding
        binding.cache_write(s["k"], s["v"], s["slots"], s["cache"])
        return s["cache"]
    kc, vc, ks, vs = s["cache"]
    ps = s["case"]["page"]
    (kc, ks), (vc, vs) = _written(s["k"], s["slots"], kc, ks, ps), _written(s["v"], s["slots"], vc, vs, ps)
    return kc, vc, ks, vs


def _run_attend(s):
    c, cache = s["case"], s["cache"]
    scale = c["dim"] ** -0.5
    if own:
        from paper_2605_00392_b200 import binding
        binding.cache_attend(s["q"], s["offsets"], s["lens"], s["table"], cache, max_q_len=s["max_q"], max_seq_len=s["max_len"], scale=scale,
                             causal=c["causal"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    off, lens, table, b, h, d = s["offsets"], s["lens"], s["table"].clamp(min=0).long(), c["batch"], c["kv_heads"], c["dim"]
    g, mq, rows = c["q_heads"] // h, s["max_q"], s["q"].shape[0]

    def pages(codes, by):                                         # [batch, kv_heads, tokens, dim]
        return (codes[table].float() * by[table][..., None, None]).transpose(1, 2).reshape(b, h, -1, d)

    n = off[1:] - off[:-1]
    at = (off[:-1, None] + torch.arange(mq, device=off.device)).clamp(max=rows - 1)
    q = s["q"].float()[at].view(b, mq, h, g, d).permute(0, 2, 3, 1, 4).reshape(b, h, g * mq, d)
    x = (q @ pages(cache[0], cache[2]).transpose(-1, -2) * scale).view(b, h, g, mq, -1)
    t = torch.arange(x.shape[-1], device=off.device)
    end = (lens - n)[:, None] + torch.arange(mq, device=off.device) + 1 if c["causal"] else lens[:, None].expand(-1, mq)
    seen = (t < end[..., None].clamp(max=lens[:, None, None]))[:, None, None]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    out = (e / total.clamp(min=1e-30)).view(b, h, g * mq, -1) @ pages(cache[1], cache[3])
    row = torch.arange(rows, device=off.device)                   # from padded places back to packed rows
    req = torch.searchsorted(off[1:].contiguous(), row.to(torch.int32), right=True)
    j = row - off[req]
    out = out.view(b, h, g, mq, d).permute(0, 3, 1, 2, 4)[req, j].reshape(rows, h * g, d)
    return out.to(torch.bfloat16), lse.permute(0, 3, 1, 2)[req, j].reshape(rows, h * g)


def work(case):
    op = case["op"]
    size = 4 if case.get("dtype") == "fp32" else 2
    if op == "rope":
        heads = case["q_heads"] + case["kv_heads"]
        return {"bytes": case["rows"] * (2 * heads * case["dim"] * size + 4), "flops": case["rows"] * heads * case["dim"] * 6}
    new, ctx = _lengths(case)
    ps, rows = case["page"], sum(new)
    pages = sum(_ceil(c + n, ps) - _ceil(c, ps) for c, n in zip(ctx, new))
    if op == "tables":
        total = rows + case["pad"]
        return {"bytes": 12 * case["batch"] + 8 * pages + 8 * total + (4 * rows if case["index"] else 0), "flops": 10 * total}
    h, d = case["kv_heads"], case["dim"]
    if op == "write":
        touched = sum(_ceil(c + n, ps) - c // ps for c, n in zip(ctx, new) if n)
        return {"bytes": 2 * rows * h * d * (size + 1) + touched * h * 16 + 4 * rows, "flops": 2 * rows * h * d * 4}
    qh, lens = case["q_heads"], [c + n for c, n in zip(ctx, new)]
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new)) if case["causal"] else sum(n * t for n, t in zip(new, lens))
    held = sum(t for n, t in zip(new, lens) if n)
    return {"bytes": rows * qh * (4 * d + 4) + 2 * held * h * d + sum(_ceil(t, ps) for t in lens) * (4 + 8 * h) + 12 * case["batch"],
            "flops": 4 * d * qh * pairs}


# ---- the definitions, in 64 bits, request by request ----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "rope": _exact_rope, "write": _exact_write, "attend": _exact_attend}[case["op"]](case, s)


def _exact_tables(case, s):
    new, ctx = _lengths(case)
    ps, table, free = case["page"], s["table"].cpu().numpy().copy(), s["free"].cpu().numpy()
    index = None if s["index"] is None else s["index"].cpu().numpy()
    base = None if s["base"] is None else s["base"].cpu().numpy()
    slots, pos = np.full(s["rows"], -1, np.int32), np.full(s["rows"], -1, np.int32)
    row, head = 0, int(s["head"][0])
    for i, (n, c) in enumerate(zip(new, ctx)):
        for p in range(_ceil(c, ps), _ceil(c + n, ps)):
            table[i, p] = free[head]
            head += 1
        x = c + np.arange(n)
        slots[row:row + n] = table[i, x // ps] * ps + x % ps
        pos[row:row + n] = x if index is None else base[i] + index[row:row + n]
        row += n
    return table, slots, pos, np.array([c + n for c, n in zip(ctx, new)], np.int32), np.array([head, 0], np.int32)


def _exact_rope(case, s):
    half, rot = case["rotary"] // 2, case["rotary"]
    freq = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(half)], dtype=torch.float64, device=s["pos"].device)
    turn = torch.polar(torch.ones_like(freq)[None, :], s["pos"].double()[:, None] * freq)[:, None, :]
    got = []
    for x, w, o in ((s["q"], s["wq"], s["q_out"]), (s["k"], s["wk"], s["k_out"])):
        y = x.double()
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * w.double()
        first, second = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["interleaved"] else (y[..., :half], y[..., half:rot])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        if case["interleaved"]:
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        else:
            y[..., :half], y[..., half:rot] = z.real, z.imag
        y[s["pos"] < 0] = o[s["pos"] < 0].double()
        got.append(y)
    return tuple(got)


def _exact_write(case, s):
    ps, slots, (kc, vc, ks, vs) = case["page"], s["slots"].cpu().numpy(), s["cache"]
    got = []
    for x, codes, scale in ((s["k"], kc, ks), (s["v"], vc, vs)):
        x, codes, scale = x.double().cpu().numpy(), codes.cpu().numpy().astype(np.float64), scale.double().cpu().numpy()
        rows = np.flatnonzero(slots >= 0)
        for part in np.split(rows, np.flatnonzero(np.diff(slots[rows] // ps)) + 1):
            if not part.size:
                continue
            p, at = slots[part[0]] // ps, slots[part] % ps
            top = np.abs(x[part]).max(axis=(0, 2))
            want = np.array([0.0 if t == 0 else 2.0 ** next(e for e in range(-160, 130) if 127 * 2.0 ** e >= t) for t in top])
            grown = np.maximum(want, scale[p] if at[0] > 0 else 0)
            shrink = np.where(grown > 0, scale[p] / np.where(grown > 0, grown, 1), 1)[:, None, None]
            codes[p][:, :at[0]] = np.rint(codes[p][:, :at[0]] * shrink)
            codes[p][:, at] = np.rint(x[part] / np.where(grown > 0, grown, 1)[None, :, None]).transpose(1, 0, 2)
            scale[p] = grown
        got += [codes.astype(np.int8), scale]
    return got[0], got[2], got[1], got[3]


def _exact_attend(case, s):
    new, ctx = _lengths(case)
    h, g, d, ps, (kc, vc, ks, vs) = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"], case["page"], s["cache"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    row = 0
    for i, (n, c) in enumerate(zip(new, ctx)):
        ids = s["table"][i, :_ceil(c + n, ps)].long()
        for a in range(h):
            k = (kc[ids, a].double() * ks[ids, a].double()[:, None, None]).reshape(-1, d)[:c + n]
            v = (vc[ids, a].double() * vs[ids, a].double()[:, None, None]).reshape(-1, d)[:c + n]
            q = s["q"][row:row + n, a * g:(a + 1) * g].double().transpose(0, 1)
            x = q @ k.T / math.sqrt(d)
            if case["causal"]:
                x = x.masked_fill(torch.ones(n, c + n, dtype=torch.bool, device=x.device).triu(c + 1), -math.inf)
            z = torch.logsumexp(x, -1)
            out[row:row + n, a * g:(a + 1) * g] = (torch.exp(x - z[..., None]) @ v).transpose(0, 1)
            lse[row:row + n, a * g:(a + 1) * g] = z.T
        row += n
    return out, lse
