"""64-bit references of the operators between pruning and the answer, written from their formulas: page tables, norms and
rotation, the 8-bit cache's codes and scales, attention over them.  Inputs and results are CPU tensors or numpy arrays."""
import math

import numpy as np
import torch


def page_map(offsets, ctx, rows, page, free, head, tables, index=None, base=None):
    """(tables, slots, positions, lens, state head) for lengths within the contract and enough pages."""
    tables, free = tables.copy(), list(free)
    slots, pos = np.full(rows, -1, np.int64), np.full(rows, -1, np.int64)
    lens = []
    for i in range(len(offsets) - 1):
        n, c = offsets[i + 1] - offsets[i], ctx[i]
        for p in range(-(-c // page), -(-(c + n) // page)):
            tables[i, p] = free[head]
            head += 1
        for j in range(n):
            row, x = offsets[i] + j, c + j
            slots[row] = tables[i, x // page] * page + x % page
            first = c if base is None else base[i]
            pos[row] = (first + index[row]) if index is not None else first + j
        lens.append(c + n)
    return tables, slots, pos, np.array(lens), head


def norm_rope(x, w, eps, positions, freq, interleaved):
    """(y, size) with size_i = |y_i| before the rotation + that of its pair's other element: what errors are relative to."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    half = freq.numel()
    angle = positions.double()[:, None, None] * freq.double()
    c, s = torch.cos(angle), torch.sin(angle)
    out, size = y.clone(), y.abs().clone()
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, size


def block_scale(top):
    if not math.isfinite(top):
        return math.nan
    if top == 0:
        return 0.0
    e = math.frexp(top)[1] - 8
    while 127 * 2.0 ** e < top:
        e += 1
    return 2.0 ** max(e, -126)


def cache_write(x, slots, codes, scales):
    """codes [pages, heads, page, dim] and scales [pages, heads] (numpy, changed in place) after rows x [rows, heads, dim]."""
    page = codes.shape[2]
    x = x.double().numpy()
    r = 0
    while r < len(slots):
        if not 0 <= slots[r] < codes.shape[0] * page:
            r += 1
            continue
        p, at, n = slots[r] // page, slots[r] % page, 1
        while r + n < len(slots) and slots[r + n] == slots[r] + n and at + n < page:
            n += 1
        for h in range(codes.shape[1]):
            new = x[r:r + n, h]
            s = block_scale(float(np.abs(new).max()))
            old = float(scales[p, h]) if at else 0.0
            s = math.nan if math.isnan(s) or math.isnan(old) else max(s, old)
            if math.isnan(s):
                codes[p, h, at:at + n] = 0
            else:
                if at and s != old:
                    codes[p, h, :at] = np.rint(codes[p, h, :at] * (old / s))
                codes[p, h, at:at + n] = np.rint(new / s) if s else 0
            scales[p, h] = s
        r += n


def attend(q, offsets, lens, tables, cache, scale, causal):
    """(out, lse, weight, dots, least) per row and head, in float64; weight = sum_t softmax_t |v_t|, dots = max_t scale sum_d |q_d k_td|,
    least = max_t (softmax_t vs_t) sum_t |vc_t|: what errors are relative to.  Rows of no request are NaN."""
    kc, vc, ks, vs = cache
    rows, heads, dim = q.shape
    group = heads // kc.shape[1]
    out = torch.full((rows, heads, dim), math.nan, dtype=torch.float64)
    lse = torch.full((rows, heads), math.nan, dtype=torch.float64)
    weight, least, dots = torch.full_like(out, math.nan), torch.full_like(out, math.nan), torch.zeros_like(lse)
    for i in range(len(lens)):
        n, L = int(offsets[i + 1] - offsets[i]), int(lens[i])
        ids = tables[i, :-(-L // kc.shape[2])].long()
        for h in range(heads):
            g = h // group
            k = (kc[ids, g].double() * ks[ids, g].double()[:, None, None]).reshape(-1, dim)[:L]
            v = (vc[ids, g].double() * vs[ids, g].double()[:, None, None]).reshape(-1, dim)[:L]
            x = q[offsets[i]:offsets[i] + n, h].double()
            s = x @ k.T * scale
            seen = torch.arange(L)[None, :] <= (L - n + torch.arange(n)[:, None] if causal else torch.full((n, 1), L))
            s = torch.where(seen, s, -math.inf)
            z = torch.logsumexp(s, -1) if L else torch.full((n,), -math.inf, dtype=torch.float64)
            p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None]), 0.0)
            r = slice(int(offsets[i]), int(offsets[i]) + n)
            # 0 * NaN of a block that a row does not see must not reach it
            out[r, h] = torch.stack([p[j, seen[j]] @ v[seen[j]] for j in range(n)]) if n else out[r, h]
            weight[r, h] = p @ v.abs().nan_to_num()
            by = vs[ids, g].double().nan_to_num().repeat_interleave(kc.shape[2])[:L]
            code = vc[ids, g].double().abs().reshape(-1, dim)[:L]
            least[r, h] = (p * by).amax(-1, keepdim=True) * (seen.double() @ code) if L else 0.0
            lse[r, h] = z
            if L:
                dots[r, h] = (x.abs() @ k.abs().T * abs(scale)).amax(-1)
    return out, lse, weight, dots, least
