"""Arguments of the binding's calls of attention: what is refused before anything is launched, and what a default stands for."""
import pytest
import torch

from paper_2406_02629_amd import P45, P61, PagedCache, SSNet


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
