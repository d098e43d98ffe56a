"""Page tables, norms and rotation, cache writes and attention over the 8-bit cache on the device, against 64-bit references.

Tolerances, from the formulas.  Whole numbers, codes and scales are exact.  Norms and rotation: the result's one rounding (half a
unit: 2^-8 of the value in bf16, 2^-24 in fp32) and fp32 arithmetic: the sum of up to 256 squares in 256 / 2 roundings at most,
root, quotient, weight, cosine and sine (an angle off by 2^-24 of a turn = 4e-7), two products: under 2e-5 of the two elements that a rotation mixes
in every case.  Attention: the output's rounding, 2^-8 of the value; a softmax weight is rounded to fp16 (2^-11 of it) and a
score is an fp32 sum of D products, off by at most D 2^-24 of sum |q_d k_td| (128: 2^-17), which moves a weight by that factor;
the sums of weights and products round in fp32 behind that (lengths up to 10^5: 2^-11 more, hardly ever that much).  A weight
times its block's scale that is under 2^-14 of the row's largest is a subnormal number of fp16, whose steps are 2^-24 of that
largest at most: off by 2^-25 of it, whatever its own size, for each token, times the token's code.  (It shows where one token has
the whole softmax and a code of 0: the element is then the sum of the others' 2^-30ths.)
"""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2605_00392_b200 import binding

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda", 0)


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


# ---- page tables ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("new,ctx,pad", [
    ([1], [0], 0), ([400], [0], 3), ([1, 1, 1], [63, 64, 65], 0), ([0, 5, 0, 0, 130, 0], [7, 0, 0, 128, 127, 16], 9),
    ([0], [5], 4), ([17] * 300, list(range(300)), 1), ([1] * 1500, [i % 200 for i in range(1500)], 5)])
@pytest.mark.parametrize("indexed", [False, True])
def test_page_map(page, new, ctx, pad, indexed):
    rng = np.random.default_rng(page + len(new))
    offsets, rows, batch = np.concatenate([[0], np.cumsum(new)]), sum(new) + pad, len(new)
    most = max(-(-(a + b) // page) for a, b in zip(new, ctx)) + 1
    ids = rng.permutation(sum(-(-(a + b) // page) for a, b in zip(new, ctx)) + 5)
    tables, used = np.full((batch, most), -7), 0
    for i, c in enumerate(ctx):
        n = -(-c // page)
        tables[i, :n] = ids[used:used + n]
        used += n
    index, base = (rng.integers(0, 4512, max(rows, 1)), rng.integers(0, 60, batch)) if indexed else (None, None)
    want = ref.page_map(offsets, ctx, rows, page, ids[used:], 2, tables, index, base)
    wide = torch.full((batch, most + 3), -9, dtype=torch.int32, device=DEV)          # table rows wider than they are long
    t = wide[:, :most]
    t.copy_(torch.from_numpy(tables))
    out = binding.PageMap.allocate(rows, batch, DEV)
    binding.map_pages(_i32(offsets), t, _i32(ids[used:]), _i32([2]), out, page_size=page, context_lens=_i32(ctx),
                      token_index=_i32(index) if indexed else None, position_base=_i32(base) if indexed else None)
    for got, w in zip((t, out.slot_map, out.positions, out.seq_lens), want):
        np.testing.assert_array_equal(got.cpu().numpy(), w)
    assert out.state.tolist() == [want[4], 0] and (wide[:, most:] == -9).all()


@pytest.mark.parametrize("batch", [5000, 6135, 6140, 6143, 6144, 16384])
def test_page_map_large_batches(batch):
    new = [i % 3 for i in range(batch)]
    off, tables = np.concatenate([[0], np.cumsum(new)]), np.full((batch, 1), -1)
    free = np.arange(batch, dtype=np.int32)[::-1].copy()
    want = ref.page_map(off, [0] * batch, sum(new), 16, free, 0, tables)
    t, out = _i32(np.full((batch, 1), -1)), binding.PageMap.allocate(sum(new), batch, DEV)
    binding.map_pages(_i32(off), t, _i32(free), _i32([0]), out, page_size=16)
    for got, w in zip((t, out.slot_map, out.positions, out.seq_lens), want):
        np.testing.assert_array_equal(got.cpu().numpy(), w)


def test_page_map_without_contexts_and_with_bases_alone():
    out = binding.PageMap.allocate(6, 2, DEV)
    t = torch.full((2, 2), -1, dtype=torch.int32, device=DEV)
    binding.map_pages(_i32([0, 2, 5]), t, _i32([3, 1]), _i32([0]), out, page_size=16, position_base=_i32([10, 20]))
    assert out.positions.tolist() == [10, 11, 20, 21, 22, -1] and out.slot_map.tolist() == [48, 49, 16, 17, 18, -1]
    assert t.tolist() == [[3, -1], [1, -1]] and out.state.tolist() == [2, 0]


def test_page_map_short_of_pages():
    # the free list ends after two of three pages: the third request gets none
    out = binding.PageMap.allocate(3, 3, DEV)
    t = torch.full((3, 1), -5, dtype=torch.int32, device=DEV)
    binding.map_pages(_i32([0, 1, 2, 3]), t, _i32([4, 6]), _i32([0]), out, page_size=16)
    assert out.slot_map.tolist() == [64, 96, -1] and t.tolist() == [[4], [6], [-1]]
    assert out.state.tolist() == [2, binding.DEV_NO_PAGES] and out.positions.tolist() == [0, 0, 0]
    # a table row too short for the second page
    t = torch.full((1, 1), -5, dtype=torch.int32, device=DEV)
    out = binding.PageMap.allocate(18, 1, DEV)
    binding.map_pages(_i32([0, 18]), t, _i32([4, 6]), _i32([0]), out, page_size=16)
    assert out.slot_map.tolist() == list(range(64, 80)) + [-1, -1] and out.state.tolist() == [2, binding.DEV_NO_PAGES]
    # a head before or behind the list
    for head in (-1, 9):
        binding.map_pages(_i32([0, 1]), t, _i32([4, 6]), _i32([head]), out, page_size=16)
        assert out.slot_map[0] == -1 and out.state[1] == binding.DEV_NO_PAGES


@pytest.mark.parametrize("offsets,ctx", [([0, 3, 1, 5], [0, 0, 0]), ([0, 2, 9, 9], [0, 0, 0]), ([0, 2, 4, 5], [0, -3, 0]),
                                         ([0, 2, 4, 5], [0, 2 ** 31 - 2, 0]), ([-4, 2, 4, 5], [0, 0, 0])])
def test_page_map_lengths_outside_the_contract(offsets, ctx):
    out = binding.PageMap.allocate(5, 3, DEV)
    t = torch.full((3, 4), -1, dtype=torch.int32, device=DEV)
    binding.map_pages(_i32(offsets), t, _i32(range(40)), _i32([0]), out, page_size=16, context_lens=_i32(ctx))
    assert out.state[1] & binding.DEV_BAD_OFFSETS
    for i in range(3):
        ok = 0 <= offsets[i] <= offsets[i + 1] <= 5 and 0 <= ctx[i] < 1000
        assert out.seq_lens[i] == (ctx[i] + offsets[i + 1] - offsets[i] if ok else 0)
        if not ok and offsets[i] >= 0:
            assert (out.slot_map[offsets[i]:max(offsets[i], min(offsets[i + 1], 5))] == -1).all()


# ---- norms and rotation ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,qh,kh,dim,rot,inter,norm,far", [
    (1, 10, 10, 128, 128, False, True, 400), (7, 3, 1, 64, 64, False, True, 5000), (33, 32, 8, 128, 64, True, True, 120000),
    (5, 2, 2, 96, 96, False, True, 100), (9, 4, 2, 256, 256, True, False, 2 ** 31 - 1), (3, 1, 1, 16, 16, False, True, 9),
    (1300, 12, 4, 80, 32, False, True, 10 ** 6), (2, 5, 1, 128, 0, False, True, 9), (4, 0, 3, 48, 32, True, True, 99),
    (3, 5, 0, 112, 112, False, True, 77), (2600, 10, 10, 128, 128, False, True, 450),
    (1000, 10, 10, 128, 128, False, True, 4000), (6100, 8, 2, 64, 32, True, True, 4000), (1023, 32, 8, 128, 128, False, False, 99)])
def test_norm_rope(dtype, rows, qh, kh, dim, rot, inter, norm, far):
    gen = torch.Generator().manual_seed(rows + dim)
    pad = 3
    x = (torch.randn(rows + pad, (qh + 2 * kh) * dim, generator=gen) * torch.exp(torch.randn(rows + pad, 1, generator=gen))).to(dtype).to(DEV)
    q, k = x[:, :qh * dim].view(rows + pad, qh, dim), x[:, qh * dim:(qh + kh) * dim].view(rows + pad, kh, dim)
    pos = torch.randint(0, far, (rows + pad,), generator=gen, dtype=torch.int64).int()
    pos[0], pos[rows - 1] = 0, far - 1
    pos[rows:] = -1
    wq = (1 + 0.3 * torch.randn(dim, generator=gen)).to(dtype).to(DEV) if norm else None
    wk = (1 + 0.3 * torch.randn(dim, generator=gen)).to(dtype).to(DEV) if norm else None
    freq = binding.rope_frequencies(rot, 1e4, DEV)
    before, keep = x.clone(), 7.0
    q_out, k_out = torch.full(q.shape, keep, dtype=dtype, device=DEV), torch.full(k.shape, keep, dtype=dtype, device=DEV)
    binding.qk_norm_rope(q, k, pos.to(DEV), freq, wq, wk, 1e-5, interleaved=inter, q_out=q_out, k_out=k_out)
    assert torch.equal(x, before)
    for t, w, got in ((q, wq, q_out), (k, wk, k_out)):
        want, size = ref.norm_rope(t.cpu(), None if w is None else w.cpu(), 1e-5, pos, freq.cpu(), inter)
        off = (got.cpu().double() - want).abs()[:rows]
        assert (off <= torch.finfo(dtype).eps / 2 * want.abs()[:rows] + 2e-5 * size[:rows]).all()
        assert (got[rows:] == keep).all()
    binding.qk_norm_rope(q, k, pos.to(DEV), freq, wq, wk, 1e-5, interleaved=inter)                 # in place, in the fused rows
    assert torch.equal(q[:rows], q_out[:rows]) and torch.equal(k[:rows], k_out[:rows])
    assert torch.equal(x[rows:], before[rows:]) and torch.equal(x[:, (qh + kh) * dim:], before[:, (qh + kh) * dim:])


@pytest.mark.parametrize("rows", [900, 4000])
def test_norm_rope_passes_over_rows_of_no_request(rows):
    # rows without a position between others, in place: left as they are, the others as without them
    q, k = (torch.randn(rows, h, 128, generator=torch.Generator(DEV).manual_seed(h), device=DEV).to(torch.bfloat16) for h in (6, 2))
    pos = torch.randint(0, 500, (rows,), generator=torch.Generator(DEV).manual_seed(1), device=DEV, dtype=torch.int32)
    holes = torch.rand(rows, generator=torch.Generator(DEV).manual_seed(2), device=DEV) < 0.4
    freq, w = binding.rope_frequencies(128, 1e4, DEV), torch.ones(128, dtype=torch.bfloat16, device=DEV)
    all_q, all_k, some_q, some_k = q.clone(), k.clone(), q.clone(), k.clone()
    binding.qk_norm_rope(all_q, all_k, pos, freq, w, w)
    binding.qk_norm_rope(some_q, some_k, torch.where(holes, -1 - pos, pos), freq, w, w)
    for before, whole, some in ((q, all_q, some_q), (k, all_k, some_k)):
        assert torch.equal(some, torch.where(holes[:, None, None], before, whole))


def test_norm_rope_zero_rows_of_zeros_and_not_finite():
    q = torch.zeros(3, 2, 64, device=DEV)
    q[1, 0, 5], q[2, 1, 9] = math.nan, math.inf
    w = torch.ones(64, device=DEV)
    o = torch.empty_like(q)
    binding.qk_norm_rope(q, q[:, :1], _i32([0, 1, 2]), binding.rope_frequencies(64, 1e4, DEV), w, None, 1e-6, q_out=o, k_out=torch.empty(3, 1, 64, device=DEV))
    assert (o[0] == 0).all() and o[1, 0].isnan().all() and (o[1, 1] == 0).all() and (o[2, 0] == 0).all() and o[2, 1].isnan().any()
    e = torch.empty(0, 2, 64, device=DEV)
    binding.qk_norm_rope(e, e, _i32([]), binding.rope_frequencies(64, 1e4, DEV))


# ---- cache writes ---------------------------------------------------------------------------------------------------

def _filled(pages, heads, page, dim, seed):
    c = binding.PagedCache.allocate(pages, heads, page, dim, DEV)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes.copy_(torch.randint(-127, 128, codes.shape, generator=gen, device=DEV))
        scale.copy_(torch.exp2(torch.randint(-9, -1, scale.shape, generator=gen, device=DEV).float()))
    return c


def _check_write(k, v, slots, cache):
    want = [t.cpu().numpy().copy() for t in cache]
    ref.cache_write(k.cpu(), slots, want[0], want[2])
    ref.cache_write(v.cpu(), slots, want[1], want[3])
    binding.cache_write(k, v, _i32(slots), cache)
    for got, w in zip(cache, want):
        np.testing.assert_array_equal(got.cpu().numpy(), w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,dim,heads,runs", [
    (16, 64, 1, [(0, 0, 1)]), (16, 128, 3, [(2, 0, 16), (1, 3, 13), (0, 15, 1)]), (64, 128, 2, [(1, 0, 64), (4, 0, 64), (2, 0, 9)]),
    (128, 128, 1, [(0, 0, 128), (3, 1, 127), (1, 100, 28)]), (128, 64, 2, [(5, 64, 64)]), (32, 64, 7, [(i, i % 32, 1) for i in range(120)]),
    (64, 128, 10, [(i, 0, 64) for i in range(90)])])
def test_cache_write(dtype, page, dim, heads, runs):
    gen = torch.Generator().manual_seed(page * dim)
    slots = [-1]
    for p, at, n in runs:
        slots += list(range(p * page + at, p * page + at + n)) + ([-1] if p % 3 == 0 else [])
    pages = max(p for p, _, _ in runs) + 2
    x = torch.randn(len(slots), 2 * heads * dim + 16, generator=gen) * torch.exp(2 * torch.randn(len(slots), 1, generator=gen))
    x = x.to(dtype).to(DEV)
    k, v = x[:, :heads * dim].view(-1, heads, dim), x[:, heads * dim:2 * heads * dim].view(-1, heads, dim)
    cache = _filled(pages, heads, page, dim, 3)
    _check_write(k, v, slots, cache)
    _check_write(v, k, slots, cache)          # and once more over what is there


def test_cache_write_token_by_token():
    cache = binding.PagedCache.allocate(2, 2, 16, 64, DEV)
    gen = torch.Generator().manual_seed(1)
    x = (torch.randn(32, 2, 64, generator=gen) * torch.exp2(torch.arange(32) % 11)[:, None, None]).to(torch.bfloat16).to(DEV)
    for t in range(32):
        _check_write(x[t:t + 1], x[31 - t:32 - t], [t], cache)


def test_cache_write_edges_of_the_scale():
    # largest values at a power of two's border, zeros, tiny ones, the type's largest, NaN and infinities
    tops = [127 / 128, 0.9922, 127.0, 127.001, 254.0, 254.01, 1e-44, 2.0 ** -126, torch.finfo(torch.float32).max, 0.0, math.nan, math.inf, -math.inf]
    cache = _filled(len(tops), 1, 16, 64, 5)
    x = torch.randn(2 * len(tops), 1, 64) * 0.1
    for i, t in enumerate(tops):
        x[2 * i:2 * i + 2] *= 0 if t == 0 else min(abs(t), 1) if math.isfinite(t) else 1
        x[2 * i + 1, 0, i] = t
    slots = [16 * i + j for i in range(len(tops)) for j in (0, 1)]
    _check_write(x.to(DEV), -x.to(DEV), slots, cache)
    # appended to: NaN stays, zero gives way, the others grow or hold
    y = torch.randn(len(tops), 1, 64)
    _check_write(y.to(DEV), y.to(DEV) * 1e-3, [16 * i + 2 for i in range(len(tops))], cache)
    _check_write(y.to(DEV), y.to(DEV), [16 * i for i in range(len(tops))], cache)      # from the first token: NaN is gone
    assert torch.isfinite(cache.k_scale).all()


def test_cache_write_slots_outside_the_cache():
    cache = _filled(2, 1, 16, 64, 6)
    x = torch.randn(5, 1, 64, device=DEV)
    _check_write(x, x, [-1, 32, 2 ** 31 - 1, 31, -2 ** 31], cache)


# ---- attention ------------------------------------------------------------------------------------------------------

def _batch(new, lens, qh, kh, dim, page, seed, spare=2):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    need = [-(-L // page) for L in lens]
    ids = torch.randperm(sum(need) + 1, generator=gen, device=DEV).int()
    tables = torch.full((len(new), max(max(need), 1)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(need):
        tables[i, :n] = ids[at:at + n]
        at += n
    cache = _filled(sum(need) + 1, kh, page, dim, seed)
    q = torch.randn(sum(new) + spare, qh, dim, generator=gen, device=DEV) * 0.4
    return q.to(torch.bfloat16), _i32(np.concatenate([[0], np.cumsum(new)])), _i32(lens), tables, cache


@pytest.fixture(params=[0, 6000], ids=["bounds", "loose"])
def bounds(request, monkeypatch):
    """max_q_len as the test has it, and far above: the bound chooses the kernel, so each test runs through both.  Gives what is added."""
    attend, space = binding.cache_attend, binding.cache_attend_workspace

    def loose(*args, max_q_len, **kw):
        return attend(*args, max_q_len=max_q_len + request.param, **kw)

    monkeypatch.setattr(binding, "cache_attend", loose)
    monkeypatch.setattr(binding, "cache_attend_workspace", lambda batch, q, *rest: space(batch, q + request.param, *rest))
    return request.param


def _check_attend(q, offsets, lens, tables, cache, max_q, max_len, scale=None, causal=True, **kw):
    keep = 3.0
    out = torch.full(q.shape, keep, dtype=torch.bfloat16, device=DEV)
    lse = torch.full(q.shape[:2], keep, device=DEV)
    binding.cache_attend(q, offsets, lens, tables, cache, max_q_len=max_q, max_seq_len=max_len, scale=scale, causal=causal, out=out,
                         lse=lse, **kw)
    dim = q.shape[2]
    want, wlse, weight, dots, least = ref.attend(q.cpu(), offsets.tolist(), lens.tolist(), tables.cpu(), [t.cpu() for t in cache],
                                          dim ** -0.5 if scale is None else scale, causal)
    n = int(offsets[-1])
    got, glse = out.cpu().double(), lse.cpu().double()
    assert (got[n:] == keep).all() and (glse[n:] == keep).all()
    want, wlse, weight, dots, least = want[:n], wlse[:n], weight[:n], dots[:n], least[:n]
    err = (2.0 ** -17 * dots)[..., None]
    off = (got[:n] - want).abs()
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -10 + 2 * err) * weight + 2.0 ** -25 * least + 1e-30
    assert (off <= bound).all(), (off / bound).max()
    empty = torch.isinf(wlse)
    assert torch.equal(glse[:n][empty], wlse[empty])
    off = (glse[:n] - wlse)[~empty].abs()
    assert (off <= err[..., 0][~empty] + 2.0 ** -20 * (1 + wlse[~empty].abs())).all()
    return out, lse


SHAPES = [
    # new, lens, query heads, kv heads, dim, page
    ([1], [1], 1, 1, 64, 16), ([1], [500], 10, 10, 128, 64), ([1, 1, 1], [16, 17, 333], 8, 1, 128, 16),
    ([1] * 9, [1, 63, 64, 65, 127, 128, 129, 0, 1000], 32, 8, 128, 64), ([1], [9000], 5, 1, 64, 128), ([1] * 70, [37 * i % 401 for i in range(70)], 12, 4, 64, 32),
    ([1], [5000], 40, 1, 128, 32), ([3, 1, 0, 8], [3, 50, 20, 700], 10, 10, 128, 64), ([5, 2], [130, 2], 16, 2, 64, 16),
    ([12, 7], [2048, 12], 7, 7, 128, 64), ([16], [16], 4, 4, 128, 128), ([64, 33], [64, 100], 8, 2, 128, 64),
    ([128], [128], 2, 2, 128, 64), ([129, 127], [129, 300], 3, 1, 64, 64), ([337, 300, 1], [350, 300, 77], 4, 4, 128, 64),
    ([260], [1300], 8, 2, 128, 32), ([700], [700], 2, 1, 64, 128), ([513], [2600], 1, 1, 128, 16), ([40, 41], [300, 41], 24, 3, 128, 16)]


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new,lens,qh,kh,dim,page", SHAPES)
def test_attend(new, lens, qh, kh, dim, page, causal):
    q, off, L, tables, cache = _batch(new, lens, qh, kh, dim, page, len(new) + lens[0])
    _check_attend(q, off, L, tables, cache, max(new), max(lens), causal=causal)


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens,qh,kh,dim,page", [
    ([3, 40], [70, 300], 160, 1, 64, 16), ([2, 0, 1], [3000, 9, 1], 512, 2, 128, 64), ([40] * 40, [40 + i for i in range(40)], 8, 8, 64, 64),
    ([40 - i for i in range(40)], [700 - 9 * i for i in range(40)], 8, 8, 128, 32), ([8] * 3, [2000, 8, 511], 1, 1, 128, 16), ([2] * 5, [513, 512, 511, 2, 5], 28, 4, 64, 64)])
def test_attend_many_heads_and_tiles(new, lens, qh, kh, dim, page):
    q, off, L, tables, cache = _batch(new, lens, qh, kh, dim, page, 31)
    _check_attend(q, off, L, tables, cache, max(new), max(lens))


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens,qh,kh,dim,page", [([1, 1], [40, 700], 8, 2, 128, 64), ([9, 5], [200, 64], 4, 4, 64, 32), ([200, 130], [333, 130], 4, 2, 128, 64)])
def test_attend_loose_bounds_strided_queries_and_scale(new, lens, qh, kh, dim, page):
    q, off, L, tables, cache = _batch(new, lens, qh, kh, dim, page, 11)
    fused = torch.randn(q.shape[0], (qh + 2 * kh) * dim, device=DEV).to(torch.bfloat16)
    part = fused[:, :qh * dim].view(-1, qh, dim)
    part.copy_(q)
    wide = torch.full((len(new), 40), -1, dtype=torch.int32, device=DEV)
    wide[:, :tables.shape[1]] = tables
    a = _check_attend(part, off, L, wide, cache, max(new) + 300, 40 * page, scale=0.31)
    _check_attend(part, off, L, wide[:, :tables.shape[1] + 1], cache, max(new), max(lens), scale=-0.2)
    # the bounds choose kernels and grids, not results beyond rounding
    b = _check_attend(q, off, L, tables, cache, max(new), max(lens), scale=0.31)
    n = int(off[-1])
    assert (a[0][:n].float() - b[0][:n].float()).abs().max() <= 2 ** -6 * b[0][:n].float().abs().max()


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens,dim", [([4], [2], 64), ([6, 1], [3, 0], 128), ([300], [200], 128), ([140, 150], [0, 129], 64)])
def test_attend_rows_that_see_nothing(new, lens, dim):
    # more queries than tokens: the first rows of a causal mask are empty
    q, off, L, tables, cache = _batch(new, lens, 4, 2, dim, 16, 5)
    out, lse = _check_attend(q, off, L, tables, cache, max(new), max(max(lens), 16))
    gap = new[0] - lens[0]
    assert (out[:gap] == 0).all() and torch.isneginf(lse[:gap]).all()


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens", [([1], [200]), ([5], [200]), ([150], [200])])
def test_attend_scales_far_apart_zero_and_large_scores(new, lens):
    q, off, L, tables, cache = _batch(new, lens, 4, 2, 128, 16, 8)
    # blocks of values 2^40 apart, and one that is all zeros: the small ones still count in the softmax's sum
    cache.v_scale[tables[0, ::2].long()] *= 2.0 ** 20
    cache.v_scale[tables[0, 1::3].long()] *= 2.0 ** -20
    cache.v_scale[tables[0, 4].long()] = 0
    cache.v[tables[0, 4].long()] = 0
    _check_attend(q, off, L, tables, cache, max(new), max(lens))
    cache.v_scale.fill_(0.01)
    cache.k_scale[tables[0, 3].long()] *= 2.0 ** 6                       # a block that takes the whole softmax
    cache.k_scale[tables[0, 5].long()] = 0
    _check_attend(q * 4, off, L, tables, cache, max(new), max(lens))
    _check_attend(torch.zeros_like(q), off, L, tables, cache, max(new), max(lens))


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new", [[1, 1], [3, 40], [150, 2]])
def test_attend_nothing_cached_and_a_scale_of_zero(new):
    q, off, L, tables, cache = _batch(new, [60, 300], 4, 2, 64, 16, 12)
    _check_attend(q, off, L, tables, cache, max(new), 300, scale=0.0, causal=False)
    lse = torch.zeros(q.shape[:2], device=DEV)
    out = binding.cache_attend(q, off, torch.zeros_like(L), tables[:, :0], cache, max_q_len=max(new), max_seq_len=0, out=torch.full_like(q, 2.0), lse=lse)
    n = sum(new)
    assert (out[:n] == 0).all() and (out[n:] == 2).all() and torch.isneginf(lse[:n]).all() and (lse[n:] == 0).all()


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens", [([1], [200]), ([5], [200]), ([150], [200])])
def test_attend_queries_of_every_size(new, lens):
    q, off, L, tables, cache = _batch(new, lens, 4, 2, 128, 64, 9)
    q = (q.float() * torch.exp2(torch.tensor([60.0, -60.0, -110.0, 100.0], device=DEV))[None, :, None]).to(torch.bfloat16)
    cache.k_scale.fill_(2.0 ** -7)
    scale = 2.0 ** -60
    _check_attend(q, off, L, tables, cache, max(new), max(lens), scale=scale)


@pytest.mark.parametrize("new,lens", [([1, 1], [100, 90]), ([6, 1], [100, 90]), ([90, 100], [100, 200])])
def test_attend_not_finite_and_pages_outside(bounds, new, lens):
    q, off, L, tables, cache = _batch(new, lens, 2, 2, 64, 16, 4)
    clean = binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens))
    last = int(L[0]) - 1

    def rows_of(t):                                # rows of request 0 that see token t
        return [j for j in range(new[0]) if lens[0] - new[0] + j >= t]

    def check(out, bad_rows, heads=(0, 1)):
        for j in range(new[0]):
            for h in (0, 1):
                if j in bad_rows and h in heads:
                    assert out[j, h].isnan().all()
                else:
                    torch.testing.assert_close(out[j, h], clean[j, h], rtol=2 ** -6, atol=1e-3)
        n = int(off[-1])
        torch.testing.assert_close(out[new[0]:n], clean[new[0]:n], rtol=2 ** -6, atol=1e-3)

    # a block of scale NaN, of keys or of values, in one head: rows that see any of its tokens; the last page's first token
    p = last // 16
    for s in (cache.k_scale, cache.v_scale):
        old = s.clone()
        s[tables[0, p].long(), 1] = math.nan
        check(binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens)), rows_of(p * 16), (1,))
        s.copy_(old)
    # table entries outside the cache
    for entry in (-1, cache.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        t = tables.clone()
        t[0, p] = entry
        check(binding.cache_attend(q, off, L, t, cache, max_q_len=max(new), max_seq_len=max(lens)), rows_of(p * 16))
    # what lies behind a sequence's end in its last page, and in pages of no request, is never used
    cache.k_scale[tables[1, -1].long() if lens[1] == max(lens) else -1].mul_(1.0)
    q2 = q.clone()
    q2[0, 0, 3] = math.inf
    o = binding.cache_attend(q2, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens))
    assert o[0, 0].isnan().all()
    torch.testing.assert_close(o[0, 1], clean[0, 1], rtol=2 ** -6, atol=1e-3)
    q2[0, 0, 3] = math.nan
    o = binding.cache_attend(q2, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens))
    assert o[0, 0].isnan().all() and not o[:int(off[-1])][1:].isnan().any()
    # lengths outside the contract
    for bad in (-1, max(lens) + 1, 2 ** 31 - 1):
        L2 = L.clone()
        L2[0] = bad
        o = binding.cache_attend(q, off, L2, tables, cache, max_q_len=max(new), max_seq_len=max(lens))
        assert o[:new[0]].isnan().all()
        torch.testing.assert_close(o[new[0]:int(off[-1])], clean[new[0]:int(off[-1])], rtol=2 ** -6, atol=1e-3)
    # a request of more rows than max_q_len is passed over; so are rows outside the tensor
    if new[0] > new[1] and bounds == 0:
        o = binding.cache_attend(q, off, L, tables, cache, max_q_len=new[1], max_seq_len=max(lens), out=torch.full_like(q, 2.0))
        assert (o[:new[0]] == 2).all()
    off2 = off.clone()
    off2[2] = q.shape[0] + 1
    o = binding.cache_attend(q, off2, L, tables, cache, max_q_len=q.shape[0], max_seq_len=max(lens), out=torch.full_like(q, 2.0))
    assert (o[new[0]:] == 2).all()


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens,qh,kh", [([1] * 5, [2000, 3, 900, 64, 4000], 8, 2), ([2, 3], [900, 40], 10, 10), ([300, 200], [400, 200], 4, 4)])
def test_attend_twice_the_same_and_across_streams_and_graphs(new, lens, qh, kh):
    q, off, L, tables, cache = _batch(new, lens, qh, kh, 128, 64, 21)
    n = int(off[-1])

    def call(stream=None, out=None):
        return binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens), stream=stream, out=out)

    a, b = call(), call()
    assert torch.equal(a[:n], b[:n])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = call(side)
    with torch.cuda.stream(side):
        d = call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a[:n], c[:n]) and torch.equal(a[:n], d[:n])
    # two graphs that share one workspace, replayed in turn
    ws = torch.empty(binding.cache_attend_workspace(len(new), max(new), max(lens), qh, kh, 128), dtype=torch.uint8, device=DEV)
    outs, graphs = [torch.zeros_like(q) for _ in range(2)], []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens), out=o, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for g, o in zip(graphs, outs):
            o.zero_()
            g.replay()
    ws.random_(0, 256)
    graphs[0].replay()
    for o in outs:
        assert torch.equal(a[:n], o[:n])


@pytest.mark.usefixtures("bounds")
def test_attend_offsets_beyond_32_bits():
    # a cache of more than 2^31 elements: pages at its end
    page, kh, dim = 128, 16, 128
    pages = 2 ** 31 // (page * kh * dim) + 40
    cache = binding.PagedCache.allocate(pages, kh, page, dim, DEV)
    ids = torch.arange(pages - 20, pages, dtype=torch.int32, device=DEV)
    rows = 20 * page - 5
    slots = (ids[:, None] * page + torch.arange(page, device=DEV, dtype=torch.int32)).flatten()[:rows].contiguous()
    k, v = (torch.randn(rows, kh, dim, device=DEV).to(torch.bfloat16) for _ in range(2))
    binding.cache_write(k, v, slots, cache)
    small = binding.PagedCache.allocate(20, kh, page, dim, DEV)
    binding.cache_write(k, v, torch.arange(rows, dtype=torch.int32, device=DEV), small)
    for a, b in zip(cache, small):
        assert torch.equal(a[-20:], b)
    for n in (1, 200):
        q = torch.randn(n, kh, dim, device=DEV).to(torch.bfloat16)
        off, L = _i32([0, n]), _i32([rows])
        a = binding.cache_attend(q, off, L, ids.view(1, -1), cache, max_q_len=n, max_seq_len=rows)
        b = binding.cache_attend(q, off, L, torch.arange(20, dtype=torch.int32, device=DEV).view(1, -1), small, max_q_len=n, max_seq_len=rows)
        assert torch.equal(a, b)


# ---- on other streams and in graphs ------------------------------------------------------------------------------------

def test_page_map_rope_and_write_in_a_graph_on_another_stream():
    """The three captured together on a stream of their own and replayed for two batches: as the same calls one by one."""
    new, ctx, page, kh, qh, dim, cap = [[5, 0, 130, 1], [1, 66, 2, 64]], [3, 64, 0, 127], 64, 2, 6, 64, 140
    off = [np.concatenate([[0], np.cumsum(n)]) for n in new]
    tables0 = torch.full((4, 6), -1, dtype=torch.int32, device=DEV)
    for i, c in enumerate(ctx):
        tables0[i, :-(-c // page)] = torch.arange(-(-c // page), device=DEV, dtype=torch.int32) + 10 + 3 * i
    free, freq = torch.arange(30, 50, device=DEV, dtype=torch.int32), binding.rope_frequencies(dim, 1e4, DEV)
    fused = [torch.randn(cap, (qh + 2 * kh) * dim, generator=torch.Generator(DEV).manual_seed(t), device=DEV).to(torch.bfloat16) for t in (0, 1)]

    def state():
        c = binding.PagedCache.allocate(60, kh, page, dim, DEV)
        for t in c:
            t.copy_(torch.randint(-99, 99, t.shape, generator=torch.Generator(DEV).manual_seed(7), device=DEV)) if t.dtype is torch.int8 else t.fill_(0.25)
        return c, tables0.clone(), binding.PageMap.allocate(cap, 4, DEV), _i32(off[0]), fused[0].clone(), _i32([2]), _i32(ctx)

    def calls(c, tables, m, offsets, x, head, lens, stream=None):
        q, k, v = (t.unflatten(1, (-1, dim)) for t in x.split([qh * dim, kh * dim, kh * dim], 1))
        binding.map_pages(offsets, tables, free, head, m, page_size=page, context_lens=lens, stream=stream)
        binding.qk_norm_rope(q, k, m.positions, freq, stream=stream)
        binding.cache_write(k, v, m.slot_map, c, stream=stream)

    eager, side = state(), torch.cuda.Stream()
    replayed = state()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        calls(*replayed, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for t in (0, 1):
        for s in (eager, replayed):
            s[3].copy_(_i32(off[t]))
            s[4].copy_(fused[t])
        calls(*eager)
        g.replay()
        for a, b in zip((*eager[0], eager[1], *eager[2], eager[4]), (*replayed[0], replayed[1], *replayed[2], replayed[4])):
            assert torch.equal(a, b)
        assert eager[2].state[1] == 0
        for s in (eager, replayed):                                     # the next batch goes behind this one
            s[5].copy_(s[2].state[:1])
            s[6].copy_(s[2].seq_lens)


@pytest.mark.parametrize("low,high", [(2 ** 31 - 1, -5), (5, 2), (-3, 2), (2, 2 ** 31 - 1), (-2 ** 31, 2 ** 31 - 1)])
def test_attend_offsets_outside_the_contract(low, high):
    # the request between two sound ones has offsets that are none: passed over, whatever the bounds allow
    q, off, L, tables, cache = _batch([2, 1, 2], [9, 9, 9], 4, 2, 64, 16, 3)
    clean = binding.cache_attend(q, off, L, tables, cache, max_q_len=2, max_seq_len=16)
    for max_q in (2, 2 ** 30, 2 ** 31 - 1):
        o = _i32([0, 2, low, high])
        got = binding.cache_attend(q, o, L, tables, cache, max_q_len=max_q, max_seq_len=16, out=torch.full_like(q, 3.0))
        torch.testing.assert_close(got[:2], clean[:2], rtol=2 ** -6, atol=1e-3)
        assert (got[5:] == 3).all()


# ---- the run of them together ---------------------------------------------------------------------------------------

def test_from_pruned_tokens_to_decode():
    """Pruning with a dynamic ratio, pages for what it keeps, norms and rotation by the kept tokens' places, the cache, prefill, then
    tokens one by one: against the formulas on what the cache holds, and the cache against what was put in."""
    from paper_2605_00392_b200 import synth
    w = synth.make("base", batch=3)
    X, offsets = w.X.to(DEV), torch.from_numpy(w.offsets).to(DEV)
    plan = binding.Plan(w.d, w.X.dtype, 3, w.total_tokens, int(np.diff(w.offsets).max()))
    run = binding.Outputs.allocate(w.total_tokens, 3, w.d, w.X.dtype, DEV)
    fields = {k: (int(v) if k in ("dynamic", "iters") else float(v)) for k, v in w.params.items()}
    plan.run(X, offsets, binding.make_params(torch.from_numpy(w.rho).to(DEV), **fields), run)
    qh, kh, dim, page, rows = 4, 2, 128, 64, w.total_tokens
    gen = torch.Generator(device=DEV).manual_seed(2)
    proj = (torch.randn(w.d, (qh + 2 * kh) * dim, generator=gen, device=DEV) * w.d ** -0.5).to(torch.bfloat16)
    wq, wk = (torch.ones(dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    freq = binding.rope_frequencies(dim, 1e4, DEV)
    cache = binding.PagedCache.allocate(40, kh, page, dim, DEV)
    tables = torch.full((3, 12), -1, dtype=torch.int32, device=DEV)
    free, head = torch.randperm(40, generator=gen, device=DEV).int(), _i32([0])
    ctx, base = _i32([0, 0, 0]), _i32([5, 0, 9])

    def step(x, off, index, max_q):
        nonlocal head, ctx
        m = binding.PageMap.allocate(x.shape[0], 3, DEV)
        binding.map_pages(off, tables, free, head, m, page_size=page, context_lens=ctx, token_index=index, position_base=base if index is not None else None)
        qkv = x @ proj
        q, k, v = (t.view(x.shape[0], -1, dim) for t in qkv.split([qh * dim, kh * dim, kh * dim], 1))
        plain = k.clone()
        binding.qk_norm_rope(q, k, m.positions, freq, wq, wk)
        binding.cache_write(k, v, m.slot_map, cache)
        n = int(off[-1])
        _, _ = _check_attend(q, off, m.seq_lens, tables, cache, max_q, 12 * page)
        got, _ = ref.norm_rope(plain[:n].cpu(), wk.cpu(), 1e-6, m.positions[:n].cpu(), freq.cpu(), False)
        s = m.slot_map[:n].long()
        held = cache.k[s // page, :, s % page].cpu().double() * cache.k_scale[s // page].cpu().double()[..., None]
        step_of = cache.k_scale[s // page].cpu().double()[..., None]
        # half a step of the code, twice where a later token made the scale grow, and the key's own rounding
        assert ((held - got).abs() <= step_of + 2 ** -8 * got.abs() + 1e-4).all()
        assert m.state[1] == 0
        head, ctx = m.state[:1].clone(), m.seq_lens.clone()
        return m

    m = step(run.Y, run.out_offsets, run.kept_idx, 400)
    counts = run.counts.tolist()
    assert m.seq_lens.tolist() == counts and (m.slot_map[sum(counts):] == -1).all()
    first = m.positions[:counts[0]].cpu().numpy()
    np.testing.assert_array_equal(first, run.kept_idx[:counts[0]].cpu().numpy() + 5)
    for t in range(3):
        step(torch.randn(3, w.d, generator=gen, device=DEV).to(torch.bfloat16), _i32([0, 1, 2, 3]), None, 1)
    assert ctx.tolist() == [c + 3 for c in counts]
