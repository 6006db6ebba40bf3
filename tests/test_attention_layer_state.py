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


def test_layers_of_a_context_never_use_a_stream_id_twice(ss):
    """the same id would share two layers' weights with the same polynomials, and mask their scores and truncations alike"""
    first, other = layer(ss), layer(ss, weight_bits=2 * ss.f)
    for at in (first, other, first, other, other):
        at.forward(x(3), {0: 3})
    ids = [i for _, i in ss.streams]
    assert len(ids) == 2 * 2 + 2 * 6 + 3 * 7 and len(set(ids)) == len(ids)


def test_ids_that_are_asked_for_are_kept_apart_from_the_others(ss):
    at = layer(ss, stream_base=1000)
    at.forward(x(1), {0: 1})
    at.forward(x(1), {0: 1})
    assert sorted({i for _, i in ss.streams}) == [998, 999] + [1000 + i for i in (0, 1, 2, 3, 4, 6)] + [1008 + i for i in (0, 1, 2, 3, 4, 6)]
    for base in (1, 993, 1000, 1017):              # weights or the first call would meet them
        with pytest.raises(ValueError):
            b = layer(ss, stream_base=base)
            b.forward(x(1), {0: 1})
    ahead = layer(ss, stream_base=1026)
    before = state(at)
    at.forward(x(1), {0: 1})                       # 1016 to 1023
    with pytest.raises(ValueError):                # 1024 and 1025 are the other's weights
        at.forward(x(1), {0: 1})
    assert state(at) != before and at.sequences.length == {0: 3}
    ahead.forward(x(1), {0: 1})


def test_ids_of_a_context():
    ss = SSNet(3, 1, device=None)
    a, b = ss.take_streams(2), ss.take_streams(8)
    assert b == a + 2 and ss.take_streams(1, first=b + 8 + 4) == b + 12
    assert ss.take_streams(5) == b + 13 and ss.take_streams(4) == b + 8 and ss.take_streams(1) == b + 18
    for first, count in ((b + 7, 1), (b + 18, 3), (a - 1, 2), (-1, 1), (1 << 64, 1), ((1 << 64) - 1, 2)):
        with pytest.raises(ValueError):
            ss.take_streams(count, first=first)
    assert ss.take_streams(2, first=a - 2) == a - 2 and ss.take_streams(1, first=0) == 0
    assert SSNet(3, 1, device=None).take_streams(1) == a
