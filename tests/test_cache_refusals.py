"""What the operators between pruning and the answer refuse, before anything is launched (no GPU needed), and the references'
own pins."""
import ctypes
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2605_00392_b200 import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 1 << 20            # an aligned address that is never followed: every call here returns before a launch


def _cache(**kw):
    c = dict(k=P, v=P, k_scale=P, v_scale=P, num_pages=8, page_size=64, kv_heads=2, head_dim=128)
    c.update(kw)
    return binding.CCache(**c)


def _map(**kw):
    a = dict(offsets=P, ctx=None, batch=2, rows=8, index=None, base=None, free=P, head=P, n_free=4, page=64, table=P, stride=4, pages=4,
             slots=P, pos=None, lens=P, state=2 * P)
    a.update(kw)
    return binding.lib().rtprune_page_map(None, *a.values())


def test_page_map_refusals():
    for bad in (dict(batch=-1), dict(rows=-1), dict(n_free=-1), dict(pages=-1), dict(stride=3), dict(offsets=None), dict(head=None),
                dict(lens=None), dict(state=None), dict(free=None), dict(table=None), dict(slots=None), dict(state=P), dict(batch=0)):
        assert _map(**bad) == INVALID, bad
    for bad in (dict(page=48), dict(page=8), dict(page=256), dict(batch=16385), dict(rows=2 ** 31 - 1)):
        assert _map(**bad) == UNSUPPORTED, bad
    assert _map(batch=0, rows=0) == OK


def _rope(**kw):
    a = dict(dtype=0, q=P, qs=256, k=P, ks=256, rows=4, qh=2, kh=2, dim=128, wq=None, wk=None, eps=1e-6, pos=P, freq=P, rot=128, inter=0,
             qo=P, qos=256, ko=P, kos=256)
    a.update(kw)
    a["eps"] = ctypes.c_float(a["eps"])
    return binding.lib().rtprune_qk_norm_rope(None, *a.values())


def test_norm_rope_refusals():
    for bad in (dict(dtype=2), dict(rows=-1), dict(qh=-1), dict(qh=0, kh=0), dict(dim=0), dict(rot=144), dict(rot=-16), dict(eps=-1.0),
                dict(eps=math.nan), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(qs=255), dict(qs=260), dict(q=P + 8),
                dict(ko=P + 2), dict(pos=None), dict(freq=None), dict(freq=P + 4), dict(wq=P + 8)):
        assert _rope(**bad) == INVALID, bad
    for bad in (dict(dim=136, rot=16), dict(rot=8), dict(dim=272, qs=544, ks=544), dict(qh=5000)):
        assert _rope(**bad) == UNSUPPORTED, bad
    assert _rope(rows=0) == OK


def _write(cache=None, **kw):
    a = dict(dtype=0, k=P, ks=256, v=P, vs=256, rows=4, slots=P)
    a.update(kw)
    return binding.lib().rtprune_cache_write(None, *a.values(), cache if cache is not None else _cache())


BAD_CACHES = [(dict(k=None), INVALID), (dict(v_scale=None), INVALID), (dict(num_pages=0), INVALID), (dict(kv_heads=0), INVALID),
              (dict(k=P + 4), INVALID), (dict(k_scale=P + 2), INVALID), (dict(page_size=48), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED),
              (dict(head_dim=96), UNSUPPORTED), (dict(num_pages=2 ** 31 // 64), UNSUPPORTED), (dict(kv_heads=1025), UNSUPPORTED)]


def test_cache_write_refusals():
    for bad in (dict(dtype=3), dict(rows=-1), dict(k=None), dict(v=None), dict(slots=None), dict(ks=128), dict(vs=258), dict(k=P + 8)):
        assert _write(**bad) == INVALID, bad
    for kw, status in BAD_CACHES:
        assert _write(_cache(**kw)) == status, kw
    assert _write(rows=2 ** 31) == UNSUPPORTED
    assert _write(rows=0) == OK


def _attend(cache=None, **kw):
    a = dict(q=P, qs=512, rows=4, heads=4, offsets=P, lens=P, batch=2, max_q=2, max_len=256, table=P, stride=4, pages=4)
    b = dict(scale=0.1, causal=1, out=P, lse=None, ws=P, bytes=1 << 30)
    for k, v in kw.items():
        (a if k in a else b)[k] = v
    b["scale"] = ctypes.c_float(b["scale"])
    return binding.lib().rtprune_cache_attend(None, *a.values(), cache if cache is not None else _cache(), *b.values())


def test_cache_attend_refusals():
    for bad in (dict(rows=-1), dict(batch=-1), dict(max_q=-1), dict(max_len=-1), dict(heads=0), dict(heads=3), dict(stride=3), dict(pages=-1),
                dict(scale=math.inf), dict(scale=math.nan), dict(max_len=257), dict(q=None), dict(offsets=None), dict(lens=None),
                dict(table=None), dict(out=None), dict(qs=511), dict(qs=516), dict(q=P + 8), dict(out=P + 4)):
        assert _attend(**bad) == INVALID, bad
    for bad in (dict(batch=65536), dict(heads=4098, qs=4098 * 128), dict(rows=2 ** 31)):
        assert _attend(**bad) == UNSUPPORTED, bad
    one = dict(num_pages=1 << 17, kv_heads=1)             # more heads than a tile has rows: the tiles of few rows, counted in 26 bits
    long = dict(num_pages=1 << 22, page_size=16, kv_heads=1)
    assert _attend(_cache(**one), heads=256, qs=256 * 128, rows=1 << 18, batch=1, max_q=1 << 18) == UNSUPPORTED
    assert _attend(_cache(**long), heads=256, qs=256 * 128, rows=1 << 17, batch=4096, max_q=1 << 17, max_len=1 << 26, pages=1 << 22,
                   stride=1 << 22) == UNSUPPORTED
    for bad in (dict(ws=None), dict(ws=P + 16), dict(bytes=0)):
        assert _attend(**bad) == WORKSPACE, bad
    for kw, status in BAD_CACHES:
        assert _attend(_cache(**kw)) == status, kw
    for nothing in (dict(rows=0), dict(batch=0), dict(max_q=0)):
        assert _attend(**nothing) == OK


def test_struct_layout():
    assert ctypes.sizeof(binding.CCache) == 56


def test_binding_checks_its_tensors():
    cpu = binding.PagedCache.allocate(4, 2, 16, 64, "cpu")
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.cache_write(q, q, i, cpu)
    with pytest.raises(ValueError):
        binding.cache_attend(q, i, i, i.view(1, 4), cpu, max_q_len=1, max_seq_len=16)
    with pytest.raises(ValueError):
        binding.qk_norm_rope(q, q, i, binding.rope_frequencies(64, 1e4, "cpu"))
    with pytest.raises(ValueError):
        binding.map_pages(i, i.view(1, 4), i, i[:1], binding.PageMap.allocate(3, 3, "cpu"), page_size=16)


def test_reference_scales():
    for top in (1e-30, 0.3, 1.0, 127 / 128, 127 / 127.999, 127.0, 127.0001, 254.0, 255.0, 3e38):
        s = ref.block_scale(top)
        assert math.frexp(s)[0] == 0.5 and 127 * s >= top > 127 * s / 2
    assert ref.block_scale(0.0) == 0 and math.isnan(ref.block_scale(math.inf)) and ref.block_scale(1e-42) == 2.0 ** -126


def test_reference_attention_is_the_mean_for_equal_scores():
    cache = binding.PagedCache.allocate(2, 1, 16, 64, "cpu")
    cache.v.random_(-127, 128)
    cache.v_scale.fill_(0.5)
    q = torch.zeros(3, 1, 64)
    out, lse, _, _, _ = ref.attend(q, [0, 3], [20], torch.tensor([[1, 0]]), cache, 1.0, True)
    v = cache.v[[1, 0], 0].double().reshape(-1, 64) * 0.5
    for j in range(3):
        assert torch.allclose(out[j, 0], v[:18 + j].mean(0)) and abs(lse[j, 0] - math.log(18 + j)) < 1e-12


def test_reference_page_map():
    t, slots, pos, lens, head = ref.page_map([0, 2, 2, 19], [15, 0, 16], 21, 16, [7, 8, 9, 5], 0, np.array([[4, -1, -1], [-1] * 3, [2, -1, -1]]))
    assert t.tolist() == [[4, 7, -1], [-1, -1, -1], [2, 8, 9]] and head == 3 and lens.tolist() == [17, 0, 33]
    assert slots[:4].tolist() == [79, 112, 128, 129] and slots[18:].tolist() == [144, -1, -1] and pos[:3].tolist() == [15, 16, 16]
