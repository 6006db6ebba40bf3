"""Which adapters an attention layer takes for its sequences.  As in test_attention_layer_state.py, without a GPU."""
import pytest
import torch

from test_attention_layer_state import layer, ss, state, x  # noqa: F401


class Places:      # of a set of adapters, what a layer asks for
    def __init__(self, adapters, K, N):
        self.adapters, self.K, self.N = adapters, K, N


def adapted(ss, qkv, out, **kw):
    asked = []

    def adapters_mod(held, x, start, index, stream_id, base, out):
        asked.append((held.adapters, index.tolist(), stream_id))
        return out

    ss.adapters_mod = adapters_mod
    at = layer(ss, stream_base=1000, adapters_qkv=qkv and Places(qkv, 8, 64), adapters_out=out and Places(out, 32, 8), **kw)
    return at, asked


@pytest.mark.parametrize("qkv,out", [(3, 3), (3, None), (None, 3), (2, 3), (3, 1)])
def test_a_place_that_no_set_has_is_refused(ss, qkv, out):
    at, asked = adapted(ss, qkv, out)
    at.forward(x(2), {7: 2}, {7: 0})
    before, noted, stream = state(at), list(ss.streams), at.stream
    for place in (3, 99, -2, 1 << 31, 1 << 40):
        with pytest.raises(ValueError, match="adapter"):
            at.forward(x(3), {7: 1, 8: 2}, {7: 1, 8: place})
        assert (state(at), ss.streams, at.stream, len(asked)) == (before, noted, stream, (qkv is not None) + (out is not None))
    # the last place of the larger set; of the sequences of other calls nothing is asked
    at.forward(x(3), {7: 1, 8: 2}, {8: 2, 50: 99})
    assert [a[:2] for a in asked[(qkv is not None) + (out is not None):]] == [(k, [-1, 2]) for k in (qkv, out) if k]


def test_sequences_without_an_adapter(ss):
    """not named, or -1"""
    at, asked = adapted(ss, 2, 2)
    at.forward(x(3), {7: 1, 8: 1, 9: 1}, {7: -1, 9: 1})
    at.forward(x(1), {7: 1}, {})
    at.forward(x(1), {7: 1})
    assert asked == [(2, [-1, -1, 1], 1008), (2, [-1, -1, 1], 1009), (2, [-1], 1018), (2, [-1], 1019)] and at.stream == 1028
