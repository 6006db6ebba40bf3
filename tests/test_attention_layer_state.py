"""What an attention layer keeps from call to call: pages and lengths of its sequences.  The kernels' place is taken by functions
that note what they are asked for, so that this runs without a GPU."""
import pytest
import torch

from paper_2406_02629_amd import SSNet, attention
from paper_2406_02629_amd import fixedpoint as fx
from paper_2406_02629_amd.attention import Attention, Sequences


class Noted(SSNet):
    """a context whose calls return tensors of the right shape and note their stream ids"""

    def __init__(self, **kw):
        super().__init__(3, 1, device=None, **kw)
        self.device, self.streams, self.appended, self.fail = torch.device("cpu"), [], [], None

    def _note(self, kind, stream_id, shape):
        if self.fail == kind:
            raise RuntimeError(kind)
        self.streams.append((kind, stream_id))
        return torch.zeros(shape, dtype=torch.int64)

    def share(self, secret, stream_id, **kw):
        return self._note("share", stream_id, (self.n,) + tuple(secret.shape))

    def pack_weights_linear(self, w):
        return w

    def linear_mod_packed(self, x, w, columns):
        return torch.zeros(x.shape[:-1] + (columns,), dtype=torch.int64)

    def degree_reduce_truncate(self, c, stream_id):
        return self._note("reduce", stream_id, c.shape)

    def truncate(self, c, stream_id):
        return self._note("truncate", stream_id, c.shape)

    def rotary_truncate(self, x, table, pos, stream_id, layout):
        return self._note("rotary", stream_id, x.shape)

    def cache_append(self, cache, k, v, slots, stream_id, table, pos, layout):
        self._note("append", stream_id, ())
        self.appended.append(slots.tolist())

    def paged_attention(self, cache, q, seq_start, block_table, ctx_len, max_ctx, stream_id, weight_bits):
        return self._note("attention", stream_id, q.shape)


class Pages:      # of a cache, what a layer asks for
    def __init__(self, ss, pages, page_size, kv_heads, dim):
        self.pages, self.page_size = pages, page_size


@pytest.fixture
def ss(monkeypatch):
    monkeypatch.setattr(attention, "PagedCache", Pages)
    return Noted()


def layer(ss, positions=200, pages=12, **kw):
    table = fx.rotary_table(positions, fx.rotary_frequencies(16), ss.f)
    return Attention(ss, torch.zeros((8, 4 * 16), dtype=torch.float64), torch.zeros((2 * 16, 8), dtype=torch.float64), 2, 1, table, pages, page_size=16, **kw)


def state(at):
    s = at.sequences
    return list(s.free), {name: list(pages) for name, pages in s.pages.items()}, dict(s.length)


def x(tokens):
    return torch.zeros((3, tokens, 8), dtype=torch.int64)


def test_a_refused_call_leaves_the_sequences_as_they_were(ss):
    at = layer(ss)
    at.forward(x(20), {0: 20})
    before = state(at)
    for counts in ({0: 7}, {0: 3, 1: 1}, {2: 30}):
        with pytest.raises(ValueError):
            at.forward(x(6), counts)
        assert state(at) == before


@pytest.mark.parametrize("kind", ["reduce", "rotary", "append", "attention"])
def test_a_call_that_fails_leaves_the_sequences_as_they_were(ss, kind):
    at = layer(ss)
    at.forward(x(20), {0: 20})
    before, ss.fail = state(at), kind
    with pytest.raises(RuntimeError):
        at.forward(x(16), {0: 14, 1: 2})
    assert state(at) == before
    ss.fail = None
    at.forward(x(16), {0: 14, 1: 2})               # the same places again
    assert ss.appended[-1] == list(range(20, 34)) + [48, 49]


def test_a_negative_number_of_tokens_is_refused(ss):
    """it would shorten a sequence and leave its pages taken"""
    at = layer(ss)
    at.forward(x(20), {0: 20})
    before = state(at)
    with pytest.raises(ValueError):
        at.sequences.extend({0: -3})
    with pytest.raises(ValueError):
        at.forward(x(2), {0: -3, 1: 5})
    assert state(at) == before
    assert at.sequences.extend({0: 0})["ctx_len"].tolist() == [20]


def test_a_sequence_does_not_outgrow_its_table(ss):
    """the kernels take the last row of the table for every position behind it"""
    at = layer(ss, positions=21)
    at.forward(x(20), {0: 20})
    before = state(at)
    for counts in ({0: 2}, {1: 1, 0: 2}, {1: 22}):
        with pytest.raises(ValueError, match="table"):
            at.forward(x(sum(counts.values())), counts)
        assert state(at) == before
    at.forward(x(22), {0: 1, 1: 21})               # up to its last row
    assert at.sequences.length == {0: 21, 1: 21}
