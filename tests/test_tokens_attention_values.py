"""Attention over values whose scales lie far apart: the weight of a key is rounded relative to the weights that its own row sees, so that no value, however large, costs
another row its bits - least of all one that the row may not see."""
import math

import pytest
import torch

from paper_2302_00282_amd import tokens as T
from test_tokens_attention import Batch, defined, queries_of, roomy, starts_of, whole


def check(batch, q, queries, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    starts = starts_of(queries)
    front = dict(prefix_table=batch.prefix_table.cuda(), prefix_length=batch.prefix) if batch.prefix else {}
    y = T.attention(q, batch.cache, batch.tables.cuda(), whole(batch.lengths), starts=whole(starts), max_queries=max(queries), scale=scale, **front)
    want, bound = defined(q, batch.cache, batch.tables, batch.lengths, starts, scale, batch.prefix_table if batch.prefix else None, batch.prefix)
    error = (y.double().cpu() - want).abs()
    assert torch.all(error <= bound), (error / bound).max()
    return y


def prompt(heads, dim, n=300, long=False, prefix=0):
    batch = Batch([n], heads, dim, 16, prefix)
    return roomy(batch) if long else batch


def slot(batch, token, b=0):
    page = batch.cache.page_tokens
    return int(batch.tables[b, token // page]), token % page


KERNELS = pytest.mark.parametrize("long", [False, True])        # (16 rows a workgroup, and 128)


@pytest.mark.gpu
@KERNELS
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_ordinary_scales(dim, long):
    check(prompt(2, dim, long=long, prefix=77), queries_of(300, 4, dim), [300])
    check(prompt(2, dim, 500, long=long), queries_of(40, 4, dim), [40])


@pytest.mark.gpu
@KERNELS
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("token", [299, 298, 128, 5])
@pytest.mark.parametrize("times", [1e3, 1e8, 1e30])
def test_a_value_does_not_reach_the_rows_before_it(times, token, dim, long):
    batch, q = prompt(2, dim, long=long), queries_of(300, 4, dim)
    alone = check(batch, q, [300])
    page, at = slot(batch, token)
    batch.cache.v_scale[page, :, at] *= times
    y = check(batch, q, [300])
    assert torch.equal(y[:token], alone[:token])                # (whatever the hidden ones hold: the very same bits)


@pytest.mark.gpu
@KERNELS
@pytest.mark.parametrize("token", [0, 60, 299])
@pytest.mark.parametrize("n", [300, 3000])
def test_a_large_value_that_is_hardly_looked_at_costs_the_others_nothing(n, token, long):
    """Its probability is e^-60 or so: times 1e8 it is nothing beside the others."""
    batch = prompt(1, 64, n, long)
    base = torch.where(queries_of(1, 1, 64)[0, 0] > 0, 1.0, -1.0)
    q = (base * 2 + 0.1 * queries_of(40, 2, 64)).bfloat16()
    page, at = slot(batch, token)
    batch.cache.k[page, 0, at] = (-127 * base).to(torch.int8)
    batch.cache.k_scale[page, 0, at] = 60 / (127 * 2 * 64 * 0.125)
    batch.cache.v_scale[page, 0, at] *= 1e8
    y = check(batch, q, [40])
    assert (y.abs() < 10).all()


@pytest.mark.gpu
@KERNELS
@pytest.mark.parametrize("prefix", [0, 5000])
def test_scales_spread_over_twelve_decades(prefix, long):
    batch = prompt(2, 64, 700, long, prefix)
    s = batch.cache.v_scale
    s *= torch.exp(torch.empty_like(s).uniform_(-13.8, 13.8, generator=torch.Generator(device="cuda").manual_seed(9)))
    check(batch, queries_of(50, 4, 64), [50])
    check(batch, queries_of(50, 4, 64, size=30.0), [50])
    check(batch, queries_of(3, 4, 64), [3])


@pytest.mark.gpu
@KERNELS
@pytest.mark.parametrize("size", [1e-30, 2e-22, 1e-10, 1e20, 5e35])
def test_scales_of_any_size(size, long):
    batch = prompt(2, 64, 130, long)
    batch.cache.v_scale *= size * 73
    check(batch, queries_of(50, 4, 64), [50])
    check(batch, queries_of(2, 4, 64, size=30.0), [2])


@pytest.mark.gpu
@KERNELS
def test_values_of_nothing_beside_large_ones(long):
    """Rows of zeros have the smallest scale there is; a key of theirs takes its share of the probability all the same."""
    batch = prompt(1, 64, 200, long)
    for t in range(0, 200, 3):
        page, at = slot(batch, t)
        batch.cache.v[page, 0, at // 16, :, at % 16] = 0
        batch.cache.v_scale[page, 0, at] = 2.0 ** -100 / 127
    check(batch, queries_of(60, 2, 64), [60])
    batch.cache.v_scale[slot(batch, 1)[0], 0, 1] *= 1e25
    check(batch, queries_of(60, 2, 64), [60])
    batch.cache.v.zero_()
    batch.cache.v_scale.masked_fill_(~torch.isnan(batch.cache.v_scale), 2.0 ** -100 / 127)
    assert not check(batch, queries_of(60, 2, 64), [60]).any()


@pytest.mark.gpu
@KERNELS
def test_scores_that_grow_from_key_to_key(long):
    """The row's reference has to follow, with small values behind large ones and the other way round."""
    for order in (1, -1):
        batch = prompt(1, 64, 400, long)
        base = torch.where(queries_of(1, 1, 64)[0, 0] > 0, 1.0, -1.0)
        q = (base + 0.05 * queries_of(40, 2, 64)).bfloat16()
        for t in range(400):
            page, at = slot(batch, t)
            batch.cache.k[page, 0, at] = (127 * base).to(torch.int8)
            batch.cache.k_scale[page, 0, at] = (t if order > 0 else 400 - t) * 0.5 / (127 * 64 * 0.125)
            batch.cache.v_scale[page, 0, at] = math.exp(-0.1 * t) if order > 0 else math.exp(0.15 * t - 30)
        check(batch, q, [40])
