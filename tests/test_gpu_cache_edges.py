"""The operators behind the pruning where what lies beside a call's data could reach its results: other rows of a tile, other requests,
shared memory of the kernel before."""
import importlib.util
import math

import pytest
import torch

import cache_ref as ref
from paper_2605_00392_b200 import binding
from test_gpu_cache_ops import DEV, _batch, _i32, bounds  # noqa: F401  (bounds: a fixture)

pytestmark = pytest.mark.gpu


# ---- attention: rows that belong to no token of the request ------------------------------------------------------------

MANY = 6000            # a bound that has calls of few rows taken by the tiles of 128 rows


def _large(q, at):
    out = q.clone()
    out[at:] = torch.where(torch.rand(out[at:].shape, generator=torch.Generator(DEV).manual_seed(3), device=DEV) < 0.5, 90.0, -90.0).to(q.dtype)
    return out


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,length,group,dim", [(100, 1500, 1, 128), (37, 900, 3, 64), (20, 1300, 5, 128), (150, 700, 1, 64), (19, 640, 7, 128)])
def test_attend_whatever_rows_lie_behind_the_request(n, length, group, dim, causal):
    q, off, L, tables, cache = _batch([n], [length], 2 * group, 2, dim, 64, n, spare=260)

    def call(x):
        return binding.cache_attend(x, off, L, tables, cache, max_q_len=MANY, max_seq_len=length, causal=causal)[:n]

    alone = call(torch.cat([q[:n], torch.zeros_like(q[n:])]))
    assert torch.equal(call(_large(q, n)), alone)
    assert torch.equal(call(torch.cat([q[:n], torch.full_like(q[n:], math.nan)])), alone)
    # as the first of two requests: the same rows, bit for bit
    both = _large(q, n)
    two = torch.cat([tables, tables])
    got = binding.cache_attend(both, _i32([0, n, n + 130]), _i32([length, length]), two, cache, max_q_len=MANY, max_seq_len=length, causal=causal)
    assert torch.equal(got[:n], alone)


@pytest.mark.parametrize("group,dim", [(3, 128), (5, 64), (7, 128), (12, 64)])
def test_attend_whatever_the_kernel_before_left_in_shared_memory(group, dim):
    # a group that does not divide 128: the last rows of a tile are never written
    n, length = 3 * (128 // group) + 1, 1500
    q, off, L, tables, cache = _batch([n], [length], 2 * group, 2, dim, 64, group)
    fill = _batch([256] * 160, [256] * 160, 1, 1, dim, 64, 2)
    got = []
    for x in (torch.zeros_like(fill[0]), _large(fill[0], 0), torch.full_like(fill[0], math.inf)):
        binding.cache_attend(x, *fill[1:], max_q_len=256, max_seq_len=256)           # every SM, every row of its tiles
        got.append(binding.cache_attend(q, off, L, tables, cache, max_q_len=MANY, max_seq_len=length)[:n])
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


# ---- attention: scales of values at the ends of their range ------------------------------------------------------------

def _check_tight(q, off, L, tables, cache, max_q, max_len, causal=True):
    """As the formulas in 64 bits, with no absolute allowance but half of bf16's smallest number, so that values of any size count.
    (Each term as in test_gpu_cache_ops: the output's rounding; weights in fp16, 2^-11, and fp32 sums; the score's error; weights that
    are subnormal in fp16.)"""
    lse = torch.zeros(q.shape[:2], device=DEV)
    out = binding.cache_attend(q, off, L, tables, cache, max_q_len=max_q, max_seq_len=max_len, causal=causal, lse=lse)
    want, wlse, weight, dots, least = ref.attend(q.cpu(), off.tolist(), L.tolist(), tables.cpu(), [t.cpu() for t in cache], q.shape[2] ** -0.5, causal)
    n = int(off[-1])
    want, wlse, weight, dots, least = want[:n], wlse[:n], weight[:n], dots[:n], least[:n]
    err = (2.0 ** -17 * dots)[..., None]
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -10 + 2 * err) * weight + 2.0 ** -25 * least + 2.0 ** -134
    got, glse = out[:n].cpu().double(), lse[:n].cpu().double()
    assert torch.isfinite(got).all() and torch.isfinite(glse).all()
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max()
    assert ((glse - wlse).abs() <= err[..., 0] + 2.0 ** -20 * (1 + wlse.abs())).all()


def _pattern(name, pages, gen):
    """log2 of each page's scale of values; None: a page of zeros."""
    at = list(range(pages))
    if name == "least":
        return [-126] * pages
    if name == "most":
        return [121] * pages
    if name == "one_ordinary":
        return [-5] + [-126] * (pages - 1)
    if name == "ordinary_last":
        return [-126] * (pages - 1) + [-5]
    if name == "zero_beside_small":
        return [None if i % 3 == 0 else -66 for i in at]
    if name == "zeros_then_least":
        return [None if i < pages // 2 else -126 for i in at]
    if name == "zeros":
        return [None] * pages
    if name == "ends":
        return [(-126, 121, -5, None)[i % 4] for i in at]
    if name == "ends_once":
        return [-126] * (pages - 1) + [121]
    return [int(x) for x in torch.randint(-126, 122, (pages,), generator=gen)]


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("name", ["least", "most", "one_ordinary", "ordinary_last", "zero_beside_small", "zeros_then_least", "zeros", "ends", "ends_once", "any"])
@pytest.mark.parametrize("new,lens,qh,kh,dim,page", [([1, 1], [1000, 77], 4, 4, 128, 16), ([5], [300], 8, 2, 64, 16), ([1], [3000], 4, 1, 128, 64),
                                                     ([20, 3], [700, 5], 4, 2, 128, 32), ([150], [640], 2, 2, 128, 16), ([140], [400], 3, 1, 64, 64)])
def test_attend_scales_at_the_ends_of_their_range(new, lens, qh, kh, dim, page, name):
    q, off, L, tables, cache = _batch(new, lens, qh, kh, dim, page, 17)
    gen = torch.Generator().manual_seed(len(name))
    for i, length in enumerate(lens):
        ids = tables[i, :-(-length // page)].long()
        for p, e in zip(ids.tolist(), _pattern(name, ids.numel(), gen)):
            cache.v_scale[p] = 0.0 if e is None else 2.0 ** e
            if e is None:
                cache.v[p] = 0
    for x in (torch.zeros_like(q), q, 8 * q):               # equal scores; ordinary ones; some 2^50 apart
        _check_tight(x, off, L, tables, cache, max(new), max(lens))


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new", [[1], [150]])
def test_attend_many_small_values_beside_an_ordinary_one(new):
    # a page of ordinary values and score 0, a thousand tokens of values near 2^-126 with a score of -6 in powers of two: 15.6 of the sum's 16.6
    q, off, L, tables, cache = _batch(new, [1024], 1, 1, 64, 16, 5)
    q.fill_(1.0)
    cache.k.fill_(-1)
    cache.k_scale.fill_(6 * math.log(2) / 64 * 8)           # q . k = -6 ln 2 / scale
    cache.v_scale.fill_(2.0 ** -126)
    first = tables[0, 0].long()
    cache.k[first], cache.v_scale[first] = 0, 2.0 ** -5
    _check_tight(q, off, L, tables, cache, max(new), 1024, causal=False)
    _check_tight(q, off, L, tables, cache, max(new), 1024)


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("x", [1.4e-36, 1e-30, 3e37])
def test_written_values_of_any_size_are_read_back(x):
    # through the cache write: rows of one value, equal scores: the value comes out
    cache = binding.PagedCache.allocate(40, 2, 16, 64, DEV)
    v = torch.full((600, 2, 64), x, device=DEV)
    binding.cache_write(torch.zeros_like(v), v, _i32(range(600)), cache)
    lse = torch.zeros(1, 2, device=DEV)
    out = binding.cache_attend(torch.zeros(1, 2, 64, dtype=torch.bfloat16, device=DEV), _i32([0, 1]), _i32([600]), _i32(range(38)).view(1, -1), cache,
                               max_q_len=1, max_seq_len=600, lse=lse)
    # half a step of the code (at least 64 of them), half a step of bf16, and the sums
    assert ((out.double() - x).abs() <= (2.0 ** -7 + 2.0 ** -8 + 2.0 ** -10) * x).all() and (lse - math.log(600)).abs().max() < 1e-4


# ---- attention: scores far below zero --------------------------------------------------------------------------------

@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new", [[1], [6], [150]])
def test_attend_scores_of_any_size_that_fp32_holds(new):
    # equal scores of -2^103 and -2^120: a row that sees them sees something
    q, off, L, tables, cache = _batch(new, [200], 4, 2, 128, 16, 6)
    cache.k.fill_(64)
    cache.v_scale.fill_(2.0 ** -4)
    for size in (60, 77):
        q.fill_(2.0 ** size)
        cache.k_scale.fill_(2.0 ** 30)
        lse = torch.zeros(q.shape[:2], device=DEV)
        out = binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=200, scale=-1.0, causal=False, lse=lse)
        n = new[0]
        ids = tables[0, :13].long()
        mean = (cache.v[ids].double().transpose(0, 1).reshape(2, -1, 128)[:, :200] / 16).mean(1).repeat_interleave(2, 0)
        # (a mean of 200 codes of equal weight: the output's rounding and the sums)
        assert ((out[:n].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -10 * 8).all()
        assert ((lse[:n].double() / -(2.0 ** (size + 43))) - 1).abs().max() < 2.0 ** -20


# ---- page tables: memory beside the outputs ----------------------------------------------------------------------------

def test_page_map_in_one_piece_of_memory():
    """All of a call's arrays back to back, and the lengths in the columns behind a table's rows: nothing overlaps, nothing is refused."""
    new, ctx, page = [5, 0, 20], [3, 16, 31], 16
    off, rows, batch = [0, 5, 5, 25], 27, 3
    arena = torch.full((4096,), -9, dtype=torch.int32, device=DEV)
    at = 0

    def take(n, values=None):
        nonlocal at
        t = arena[at:at + n]
        at += n
        if values is not None:
            t.copy_(_i32(values))
        return t

    o, c, free, head = take(4, off), take(3, ctx), take(6, [9, 8, 7, 6, 5, 4]), take(1, [1])
    slots, pos, lens, state = take(27), take(27), take(3), take(2)
    take(-at % 4)                                                          # (16-byte stores of rows need it)
    wide = take(3 * 8).view(3, 8)
    tables = wide[:, :5]
    tables.copy_(_i32([[0, -1, -1, -1, -1], [1, -1, -1, -1, -1], [2, 3, -1, -1, -1]]))
    base = wide[1, 5:]                                                     # a row's unused columns
    base.copy_(_i32([100, 200, 300]))
    want = ref.page_map(off, ctx, rows, page, [9, 8, 7, 6, 5, 4], 1, tables.cpu().numpy(), None, [100, 200, 300])
    binding.map_pages(o, tables, free, head, (slots, pos, lens, state), page_size=page, context_lens=c, position_base=base)
    for got, w in zip((tables, slots, pos, lens), want):
        assert got.tolist() == w.tolist()
    assert state.tolist() == [want[4], 0] and base.tolist() == [100, 200, 300] and (arena[at:] == -9).all()


def test_page_map_refuses_its_own_lengths_as_contexts():
    # the decode loop that hands one step's lengths to the next in place
    m = binding.PageMap.allocate(3, 3, DEV)
    m.seq_lens.fill_(15)
    t, off, free = torch.full((3, 4), 1, dtype=torch.int32, device=DEV), _i32([0, 1, 2, 3]), _i32([5, 6, 7, 8])
    for bad in (dict(context_lens=m.seq_lens), dict(position_base=m.seq_lens), dict(token_index=m.positions)):
        with pytest.raises(binding.RtpruneError):
            binding.map_pages(off, t, free, _i32([0]), m, page_size=16, **bad)
    with pytest.raises(binding.RtpruneError):
        binding.map_pages(off, t, free, m.state[1:], m, page_size=16)
    assert m.seq_lens.tolist() == [15] * 3


@pytest.mark.parametrize("page,batch", [(16, 3), (64, 700)])
def test_page_map_decode_loop_with_two_maps_in_turn(page, batch):
    """Tokens one by one, the lengths of one map the contexts of the other: every token has a slot of its own, in order."""
    maps = [binding.PageMap.allocate(batch, batch, DEV) for _ in range(2)]
    off = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    tables = torch.full((batch, 5), -1, dtype=torch.int32, device=DEV)
    free = torch.arange(5 * batch, dtype=torch.int32, device=DEV).flip(0).contiguous()
    maps[1].seq_lens.copy_(torch.arange(batch, device=DEV) % 3)
    maps[1].state.zero_()
    taken = sum(1 for i in range(batch) if i % 3)                          # pages for the tokens that are there
    tables[maps[1].seq_lens > 0, 0] = free[:taken]
    maps[1].state[0] = taken
    seen = set()
    for t in range(2 * page + 3):
        m, before = maps[t % 2], maps[(t + 1) % 2]
        binding.map_pages(off, tables, free, before.state[:1], m, page_size=page, context_lens=before.seq_lens)
        x = before.seq_lens.long()
        assert m.state[1] == 0 and torch.equal(m.seq_lens, before.seq_lens + 1) and torch.equal(m.positions.long(), x)
        assert torch.equal(m.slot_map.long(), tables.long()[torch.arange(batch, device=DEV), x // page] * page + x % page)
        slots = m.slot_map.tolist()
        assert not seen & set(slots) and len(set(slots)) == batch
        seen |= set(slots)


def test_page_map_of_no_requests():
    # the free list goes on from where it was
    m = binding.PageMap.allocate(0, 0, DEV)
    m.state.fill_(77)
    side = torch.cuda.Stream()
    for stream in (None, side):
        side.wait_stream(torch.cuda.current_stream())
        binding.map_pages(_i32([0]), torch.empty(0, 4, dtype=torch.int32, device=DEV), _i32([5, 6]), _i32([1]), m, page_size=16, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        assert m.state.tolist() == [1, 0]
        m.state.fill_(77)


def test_page_map_again_after_too_short_a_row():
    """RTPRUNE_DEV_NO_PAGES: the call repeated from the old head, with rows that are wide enough, is as if the first had not been."""
    off, ctx, free = _i32([0, 40, 45]), _i32([3, 0]), _i32([9, 8, 7, 6])
    wide = torch.full((2, 4), -1, dtype=torch.int32, device=DEV)
    wide[0, 0] = 2
    one, m = wide.clone(), binding.PageMap.allocate(45, 2, DEV)
    binding.map_pages(off, wide[:, :2], free, _i32([0]), m, page_size=16, context_lens=ctx)
    # the second request's page comes behind both of the first's, of which its row could take one
    assert m.state.tolist() == [3, binding.DEV_NO_PAGES] and wide.tolist() == [[2, 9, -1, -1], [7, -1, -1, -1]]
    assert (m.slot_map[29:40] == -1).all() and m.slot_map[40] == 7 * 16
    binding.map_pages(off, wide, free, _i32([0]), m, page_size=16, context_lens=ctx)
    once = binding.PageMap.allocate(45, 2, DEV)
    binding.map_pages(off, one, free, _i32([0]), once, page_size=16, context_lens=ctx)
    assert torch.equal(wide, one) and all(torch.equal(a, b) for a, b in zip(m, once)) and m.state.tolist() == [3, 0]


# ---- attention: waits that give up -------------------------------------------------------------------------------------

@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens,qh,kh,dim,page", [
    ([1], [500], 2, 2, 128, 64), ([1], [9000], 4, 1, 64, 128), ([1] * 70, [37 * i % 401 for i in range(70)], 12, 4, 64, 32),
    ([3, 0, 5], [700, 9, 40], 8, 2, 128, 16), ([300, 0, 77], [2000, 0, 100], 3, 1, 64, 64), ([260] * 40, [300 + i for i in range(40)], 8, 8, 128, 64)])
def test_attend_waits_that_give_up_leave_nan_and_no_trace(new, lens, qh, kh, dim, page, monkeypatch):
    q, off, L, tables, cache = _batch(new, lens, qh, kh, dim, page, 3)
    n = int(off[-1])

    def call():
        out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device=DEV)
        binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens), out=out, lse=lse)
        return out, lse

    clean = call()
    lib = binding.lib()
    with monkeypatch.context() as m:
        m.setattr(lib, "rtprune_cache_attend", lambda *args: lib.rtprune_test_cache_attend_expired(*args, polls))
        for polls in (0, 1, 1, 2, 2, 3, 5):
            out, lse = call()
            gone = out[:n].isnan().all(-1)
            # a row is there, bit for bit, or gone
            assert polls > 0 or gone.all()
            assert torch.equal(gone, out[:n].isnan().any(-1)) and torch.equal(gone, lse[:n].isnan())
            assert torch.equal(out[:n][~gone], clean[0][:n][~gone]) and torch.equal(lse[:n][~gone], clean[1][:n][~gone])
            assert (out[n:] == 3).all() and (lse[n:] == 3).all()
    for a, b in zip(call(), clean):
        assert torch.equal(a, b) and not a.isnan().any()


# ---- sizes of a serving batch ----------------------------------------------------------------------------------------

def _check(q, off, L, tables, cache, max_q, max_len, rows):
    """Some of the requests against the formulas, one by one."""
    lse = torch.zeros(q.shape[:2], device=DEV)
    out = binding.cache_attend(q, off, L, tables, cache, max_q_len=max_q, max_seq_len=max_len, lse=lse)
    host = [t.cpu() for t in cache]
    for i in rows:
        a, b = int(off[i]), int(off[i + 1])
        want, wlse, weight, dots, least = ref.attend(q[a:b].cpu(), [0, b - a], [int(L[i])], tables[i:i + 1].cpu(), host, q.shape[2] ** -0.5, True)
        err = (2.0 ** -17 * dots)[..., None]
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -10 + 2 * err) * weight + 2.0 ** -25 * least + 1e-30
        assert ((out[a:b].cpu().double() - want).abs() <= bound).all(), i
        off_lse = (lse[a:b].cpu().double() - wlse).abs()
        assert ((off_lse <= err[..., 0] + 2.0 ** -20 * (1 + wlse.abs())) | torch.isneginf(wlse)).all(), i


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("batch", [161, 256, 700, 4001])
def test_attend_more_requests_than_threads_of_a_block(batch):
    # a token of each, of lengths from nothing to several blocks, some requests without a row
    new, lens = [int(i % 11 != 3) for i in range(batch)], [(i * 53) % 390 for i in range(batch)]
    q, off, L, tables, cache = _batch(new, lens, 8, 2, 64, 16, batch)
    _check(q, off, L, tables, cache, 1, 390, list(range(0, batch, 37)) + [batch - 1])


@pytest.mark.usefixtures("bounds")
def test_attend_more_requests_than_threads_of_several_rows():
    new, lens = [(i * 7) % 5 for i in range(500)], [20 + (i * 29) % 900 for i in range(500)]
    q, off, L, tables, cache = _batch(new, lens, 4, 4, 128, 64, 9)
    _check(q, off, L, tables, cache, 4, 920, range(0, 500, 23))


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new", [1, 3, 40])
def test_attend_a_context_of_100000_tokens(new):
    q, off, L, tables, cache = _batch([new, 1], [100003, 60], 8, 1, 128, 128, 4)
    _check(q, off, L, tables, cache, new, 100003, [0, 1])


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("new,lens", [([1, 1], [100, 90]), ([6, 1], [100, 37]), ([90, 100], [100, 203])])
def test_attend_reads_nothing_behind_a_length(new, lens):
    """Codes behind a request's last token, in its last page, and the codes and scales of pages that are nobody's: whatever they are."""
    q, off, L, tables, cache = _batch(new, lens, 2, 2, 64, 16, 4)
    n = sum(new)

    def call():
        lse = torch.zeros(q.shape[:2], device=DEV)
        return binding.cache_attend(q, off, L, tables, cache, max_q_len=max(new), max_seq_len=max(lens), lse=lse)[:n], lse[:n]

    clean = call()
    used = torch.zeros(cache.k.shape[0], dtype=torch.bool, device=DEV)
    for i, length in enumerate(lens):
        used[tables[i, :-(-length // 16)].long()] = True
        last = tables[i, (length - 1) // 16].long()
        for codes in (cache.k, cache.v):
            codes[last, :, (length - 1) % 16 + 1:] = 127 if i else -127
    assert not used.all()
    for codes in (cache.k, cache.v):
        codes[~used] = 127
    for scale in (cache.k_scale, cache.v_scale):
        scale[~used] = math.nan
    for a, b in zip(call(), clean):
        assert torch.equal(a, b)


@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("low,high", [(-60, 20), (-60, -50), (10, 20), (-61, 21)])
@pytest.mark.parametrize("new,lens,causal", [([1, 3], [700, 65], True), ([150], [400], True), ([40, 9], [40, 9], True), ([150, 20], [300, 77], False)])
def test_attend_scales_about_the_border_of_one_reference(new, lens, causal, low, high):
    # no zeros: what has m' as the reference of its sum, through blocks seen in part
    q, off, L, tables, cache = _batch(new, lens, 4, 2, 64, 16, 23)
    cache.v_scale.copy_(torch.exp2(torch.randint(low, high + 1, cache.v_scale.shape, generator=torch.Generator().manual_seed(1)).float()))
    for x in (q, 8 * q):
        _check_tight(x, off, L, tables, cache, max(new), max(lens), causal)


def test_calls_without_the_quick_ways_to_device_and_stream(monkeypatch):
    # a torch that has not got them
    with monkeypatch.context() as m:
        for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
            m.delattr(torch._C, name)
        spec = importlib.util.find_spec(binding.__name__)
        plain = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(plain)
    assert plain._current_device is torch.cuda.current_device and binding._current_device is not torch.cuda.current_device
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert plain._current_stream(0) == binding._current_stream(0) == side.cuda_stream
    q, off, L, tables, cache = _batch([2], [40], 2, 2, 64, 16, 1)
    a, b = (x.cache_attend(q, off, L, tables, cache, max_q_len=2, max_seq_len=40) for x in (plain, binding))
    assert torch.equal(a, b)


# ---- attention: batches padded with requests that have no rows --------------------------------------------------------------

@pytest.mark.usefixtures("bounds")
@pytest.mark.parametrize("batch", [40, 256, 4097, 65535])
@pytest.mark.parametrize("where", ["behind", "ahead", "between", "spread"])
def test_attend_padded_batches(batch, where):
    real = [(1, 700), (3, 64), (1, 1), (2, 900), (1, 0), (4, 300), (1, 129), (1, 517)]
    at = {"behind": range(8), "ahead": range(batch - 8, batch), "between": [0, 1, 2, 3, batch - 4, batch - 3, batch - 2, batch - 1],
          "spread": range(0, batch // 8 * 8, batch // 8)}[where]
    new, lens = [0] * batch, [0] * batch
    for i, (n, length) in zip(at, real):
        new[i], lens[i] = n, length
    q, off, L, tables, cache = _batch([n for n, _ in real], [x for _, x in real], 6, 2, 128, 64, 3)
    padded = torch.full((batch, tables.shape[1]), -1, dtype=torch.int32, device=DEV)
    padded[list(at)] = tables
    got = []
    for o, lengths, t in ((off, L, tables), (_i32([0] + torch.tensor(new).cumsum(0).tolist()), _i32(lens), padded)):
        lse = torch.full(q.shape[:2], 3.0, device=DEV)
        out = binding.cache_attend(q, o, lengths, t, cache, max_q_len=4, max_seq_len=900, out=torch.full_like(q, 3.0), lse=lse)
        got.append((out, lse))
    want, wlse, weight, dots, least = ref.attend(q.cpu(), off.tolist(), L.tolist(), tables.cpu(), [t.cpu() for t in cache], 128 ** -0.5, True)
    n = int(off[-1])
    err = (2.0 ** -17 * dots[:n])[..., None]
    bound = 2.0 ** -8 * want[:n].abs() + (2.0 ** -10 + 2 * err) * weight[:n] + 2.0 ** -25 * least[:n] + 1e-30
    empty = torch.isinf(wlse[:n])
    for out, lse in got:
        assert ((out[:n].cpu().double() - want[:n]).abs() <= bound).all() and (out[n:] == 3).all()
        assert torch.equal(torch.isneginf(lse[:n].cpu()), empty) and (lse[n:] == 3).all()
        assert ((lse[:n].cpu().double() - wlse[:n])[~empty].abs() <= err[..., 0][~empty] + 2.0 ** -20 * (1 + wlse[:n][~empty].abs())).all()
