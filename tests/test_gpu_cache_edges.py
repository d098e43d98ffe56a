"""The operators behind the pruning where what lies beside a call's data could reach its results: other rows of a tile, other requests,
shared memory of the kernel before."""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2605_00392_b200 import binding
from test_gpu_cache_ops import DEV, _batch, _i32, bounds  # noqa: F401  (a fixture)

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
