"""Arguments of the binding's calls of attention: what is refused before anything is launched, and what a default stands for."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, PagedCache, SSNet
from paper_2406_02629_amd import fixedpoint as fx
from paper_2406_02629_amd.attention import Attention
from test_attention import Context, host


def cache_like(ss, heads=2, dim=32):
    """what the binding reads of a cache of `ss`, without memory on a GPU"""
    cache = PagedCache.__new__(PagedCache)
    cache.n, cache.p, cache.pages, cache.page_size, cache.heads, cache.head_dim = ss.n, ss.p, 1, 16, heads, dim
    return cache


@pytest.mark.parametrize("other", [dict(n=3, t=1, p=P45), dict(n=4, t=1, p=P61)])
def test_a_cache_of_another_field_or_scheme_is_refused(other):
    """its pages have another size, so that the library would read and write past their end: digits of 8 bits to an element, 8 over 2^61 - 1 and 6 over
    2^45 - 55"""
    ss, theirs = SSNet(3, 1, device=None), SSNet(device=None, **other)
    sizes = [s.lib.ssnet_cache_page_bytes(s._ctx, 16, 2, 32) for s in (ss, theirs)]
    assert sizes[0] != sizes[1]
    x, start = torch.zeros((3, 1, 2, 32), dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    for net, cache in ((ss, cache_like(theirs)), (theirs, cache_like(ss))):
        with pytest.raises(ValueError, match="cache"):
            net.cache_append(cache, x, x, torch.zeros(1, dtype=torch.int64), 0)
        with pytest.raises(ValueError, match="cache"):
            net.paged_attention(cache, x, start, torch.zeros((1, 1), dtype=torch.int32), start[:1], 1, 0)


@pytest.mark.gpu
def test_a_cache_knows_its_field():
    for p in (P61, P45):
        assert PagedCache(SSNet(3, 1, p=p), 1, 16, 1, 16).p == p


@pytest.mark.parametrize("p,f", [(P61, 13), (P45, 12), (P61, 10)])
def test_short_weights_are_the_default_while_they_sum_to_one(p, f):
    """Scores of unit variance.  A weight is rounded to a multiple of 2^-f.  At 2^(f-2) keys the mean weight is 4 units and those that round to 0
    (below half a unit, an eighth of the mean) are exp(x - 1/2) < 1/8 with x normal: 5.7 % of the keys, 0.5 % of the sum, of which the keys just above half a unit, that
    round up, give back most; the other roundings add up to sqrt(2^(f-2) / 12) units, 0.45 % of the sum at f = 10 and less above.  So 1 %
    is the bound at the limit, while four times as many keys lose more than 4 % (keys below half of the mean weight: 42 % of them, 12 % of the sum)."""
    ss = SSNet(3, 1, f=f, p=p, device=None)
    limit = 1 << (f - 2)
    assert ss.short_weights_serve(limit) and not ss.short_weights_serve(limit + 1) and ss.short_weights_serve(1)

    def total(keys):
        s = (np.random.default_rng(keys).standard_normal(keys) * 4.0 ** f).astype(np.int64)
        return orc.softmax_row((s % p).astype(np.uint64), f, round(math.log2(math.e) * 2 ** 24), f, p).sum() / 2 ** f

    assert abs(total(limit) - 1) < 0.01 and total(4 * limit) < 0.96


@pytest.mark.parametrize("p,f", [(P61, 13), (P45, 12)])
def test_a_long_context_needs_its_weight_bits_given(p, f):
    ss = SSNet(3, 1, f=f, p=p, device=None)
    x, start = torch.zeros((3, 1, 2, 32), dtype=torch.int64), torch.zeros(2, dtype=torch.int32)

    def call(max_ctx, **kw):
        ss.paged_attention(cache_like(ss), x, start, torch.zeros((1, 1), dtype=torch.int32), start[:1], max_ctx, 0, **kw)

    with pytest.raises(ValueError, match="weight_bits"):
        call((1 << (f - 2)) + 1)
    for kw in (dict(max_ctx=1 << (f - 2)), dict(max_ctx=1 << f, weight_bits=f), dict(max_ctx=1 << f, weight_bits=2 * f)):
        with pytest.raises(TypeError):             # goes on, to the tensors that are not on a GPU
            call(**kw)


@pytest.mark.gpu
def test_default_weight_bits():
    c = Context(3, 1, P61, 13, [1], [40], 2, 1, 16, 16)
    assert torch.equal(c.run(None, max_ctx=2048), c.run(13)) and np.array_equal(host(c.run(None)), c.want(13))
    ss, out = c.ss, torch.zeros((3, 1, 2, 16), dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        c.run(None, max_ctx=2049, out=out)
    assert not out.any()
    w_qkv, w_out = torch.zeros((8, 4 * 16), dtype=torch.float64), torch.zeros((2 * 16, 8), dtype=torch.float64)
    for positions, pages, bits in ((2048, 200, 13), (4096, 128, 13), (2049, 200, 26), (2048, 1, 13)):
        table = fx.rotary_table(positions, fx.rotary_frequencies(16), 13).cuda()
        assert Attention(ss, w_qkv, w_out, 2, 1, table, pages, page_size=16).bits == bits
    assert Attention(ss, w_qkv, w_out, 2, 1, table, 200, page_size=16, weight_bits=13).bits == 13


@pytest.mark.parametrize("scale,taken", [(0.0, False), (-1.0, False), (0.0027, False), (0.0028, True), (2.77, True), (2.78, False), (3.0, False), (4.0, False),
                                         (math.inf, False), (math.nan, False)])
def test_factors_of_the_scores_are_those_that_the_library_takes(scale, taken):
    """2^16 <= round(2^24 log2(e) scale) < 2^26"""
    ss = SSNet(3, 1, device=None)
    x, start = torch.zeros((3, 1, 2, 32), dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    assert taken == (math.isfinite(scale) and 1 << 16 <= round(scale * math.log2(math.e) * 2 ** 24) < 1 << 26)
    with pytest.raises(TypeError if taken else ValueError):      # (goes on, to the tensors that are not on a GPU)
        ss.paged_attention(cache_like(ss), x, start, torch.zeros((1, 1), dtype=torch.int32), start[:1], 1, 0, scale=scale)
