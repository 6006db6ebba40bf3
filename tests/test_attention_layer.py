"""A whole attention layer on shares (dense layers, rotary positions, paged cache, attention) against the same layer in plain whole numbers:
every step opens to what it computes, so the opened result has to be equal, however the tokens are cut into chunks."""
import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, PagedCache, SSNet
from paper_2406_02629_amd import fixedpoint as fx
from paper_2406_02629_amd.attention import Attention, Sequences
from test_attention import fixed_scale, host

gpu = pytest.mark.gpu


class _Pages:      # of a cache, what Sequences asks for
    pages, page_size = 5, 16


def test_pages_are_given_and_taken_back():
    s = Sequences(_Pages())
    b = s.extend({7: 16, 3: 1})
    assert b["pos"].tolist() == list(range(16)) + [0] and b["seq_start"].tolist() == [0, 16, 17] and b["ctx_len"].tolist() == [16, 1]
    assert b["slots"].tolist() == list(range(16)) + [16] and b["max_ctx"] == 16
    b = s.extend({3: 2, 7: 1})
    assert b["pos"].tolist() == [1, 2, 16] and b["block_table"].tolist() == [[1, 0], [0, 2]] and b["slots"].tolist() == [17, 18, 32]
    with pytest.raises(MemoryError):
        s.extend({3: 46})
    assert s.length == {7: 17, 3: 3} and len(s.free) == 2
    s.release(7)
    assert len(s.free) == 4 and s.extend({3: 46, 9: 0})["ctx_len"].tolist() == [49, 0]


class Plain:
    """the layer in whole numbers"""

    def __init__(self, w_qkv, w_out, heads, kv, table, f, bits, p, layout):
        self.w_qkv, self.w_out = (np.rint(w * 2 ** f).astype(np.int64) for w in (w_qkv, w_out))
        self.heads, self.kv, self.table, self.f, self.bits, self.p, self.layout = heads, kv, table.astype(np.int64), f, bits, p, layout
        self.dim = w_out.shape[0] // heads
        self.k, self.v = {}, {}

    def turned(self, x, pos):
        half = self.table.shape[1]
        out = x.copy()
        a, b = (np.arange(half), np.arange(half) + half) if self.layout == "half" else (2 * np.arange(half), 2 * np.arange(half) + 1)
        c, s = self.table[pos, :, 0], self.table[pos, :, 1]
        out[:, a], out[:, b] = (x[:, a] * c - x[:, b] * s) >> self.f, (x[:, b] * c + x[:, a] * s) >> self.f
        return out

    def token(self, name, x):
        """one token of a sequence, x [width] whole numbers"""
        f = self.f
        y = ((x @ self.w_qkv) >> f).reshape(-1, self.dim)
        ks, vs = self.k.setdefault(name, []), self.v.setdefault(name, [])
        pos = len(ks)
        q = self.turned(y[:self.heads], pos)
        ks.append(self.turned(y[self.heads:self.heads + self.kv], pos))
        vs.append(y[self.heads + self.kv:])
        k, v, out = np.array(ks), np.array(vs), []
        for h in range(self.heads):
            g = h // (self.heads // self.kv)
            w = orc.softmax_row(((k[:, g] @ q[h]) % self.p).astype(np.uint64), f, fixed_scale(self.dim), self.bits, self.p).astype(np.int64)
            out.append(w @ v[:, g])
        o = np.concatenate(out) >> f
        if self.bits == 2 * f:
            o >>= f
        return (o @ self.w_out) >> f


@gpu
@pytest.mark.parametrize("n,t,p,f,bits,layout,heads,kv,dim,rot,page", [
    (3, 1, P61, 13, 26, "half", 4, 2, 32, 32, 16), (5, 2, P61, 13, 13, "interleaved", 4, 1, 48, 24, 32), (3, 1, P45, 12, 12, "half", 2, 2, 64, 64, 16),
    (7, 3, P61, 12, 24, "half", 6, 2, 16, 16, 48)])
def test_layer_opens_to_the_plain_layer_however_tokens_are_cut(n, t, p, f, bits, layout, heads, kv, dim, rot, page):
    rng = np.random.default_rng(4)
    width = 40
    w_qkv, w_out = rng.standard_normal((width, (heads + 2 * kv) * dim)) / width ** 0.5, rng.standard_normal((heads * dim, width)) / (heads * dim) ** 0.5
    table = fx.rotary_table(200, fx.rotary_frequencies(rot, factor=2.0, original=64), f)
    tokens = {0: rng.standard_normal((37, width)), 1: rng.standard_normal((70, width)), 2: rng.standard_normal((3, width))}
    plain = Plain(w_qkv, w_out, heads, kv, table.numpy(), f, bits, p, layout)
    want = {s: np.array([plain.token(s, np.rint(x * 2 ** f).astype(np.int64)) for x in xs]) for s, xs in tokens.items()}
    for cuts in ([{0: 37, 1: 70, 2: 3}], [{0: 20, 1: 1}, {1: 50, 0: 1, 2: 2}, {0: 1, 1: 1, 2: 1}, {1: 17, 0: 14}, {0: 1, 1: 1}]):
        ss = SSNet(n, t, f=f, seed=3, p=p)
        layer = Attention(ss, torch.from_numpy(w_qkv), torch.from_numpy(w_out), heads, kv, table.cuda(), pages=12, page_size=page, layout=layout,
                          weight_bits=bits)
        done = {s: 0 for s in tokens}
        for stream, counts in enumerate(cuts):
            x = np.concatenate([tokens[s][done[s]:done[s] + c] for s, c in counts.items()])
            shares = ss.share(fx.encode(torch.from_numpy(x).cuda(), f, p), stream_id=100 + stream)
            y = layer.forward(shares, counts)
            assert y.shape == shares.shape
            got = fx.lift(ss.reconstruct(y, list(range(n - t, n + 1))), p).cpu().numpy()
            at = 0
            for s, c in counts.items():
                assert np.array_equal(got[at:at + c], want[s][done[s]:done[s] + c]), (s, done[s])
                done[s] += c
                at += c
        assert all(done[s] == len(tokens[s]) for s in tokens)


@gpu
def test_refusals_of_the_binding():
    ss = SSNet(3, 1)
    cache = PagedCache(ss, 2, 16, 2, 32)
    x = torch.zeros((3, 4, 2, 32), dtype=torch.int64, device="cuda")
    table, pos = torch.zeros((8, 16, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    slots = torch.arange(4, device="cuda")
    start, tab, ln = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 4], [[0]], [4]))
    for call in (lambda: ss.rotary_truncate(x.float(), table, pos, 0), lambda: ss.rotary_truncate(x.transpose(1, 2), table, pos, 0),
                 lambda: ss.rotary_truncate(x, table.long(), pos, 0), lambda: ss.rotary_truncate(x[:, ::2], table, pos[:2].long(), 0),
                 lambda: ss.cache_append(cache, x, x.cpu(), slots, 0), lambda: ss.cache_append(cache, x, x, slots.int(), 0),
                 lambda: ss.paged_attention(cache, x, start.long(), tab, ln, 4, 0), lambda: ss.rotary_truncate(x, table, pos, 0, out=x.cpu())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ss.rotary_truncate(x[:2], table, pos, 0), lambda: ss.rotary_truncate(x, table[..., 0].contiguous(), pos, 0),
                 lambda: ss.rotary_truncate(x, table, pos, 0, layout="quarter"), lambda: ss.rotary_truncate(x, table, pos[:3].contiguous(), 0),
                 lambda: ss.cache_append(cache, x, x, slots, 0, table=table), lambda: ss.cache_append(cache, x[:, :, :1], x[:, :, :1], slots, 0),
                 lambda: ss.paged_attention(cache, x, start, tab[0], ln, 4, 0), lambda: ss.paged_attention(cache, x, start[:1], tab, ln, 4, 0),
                 lambda: ss.paged_attention(cache, x, start, tab, ln, 4, 0, scale=0.0),
                 lambda: Attention(ss, torch.zeros(8, 7), torch.zeros(64, 8), 2, 2, table, 2),
                 lambda: Attention(ss, torch.zeros(8, 192), torch.zeros(64, 8), 2, 2, table, 2, weight_bits=20)):
        with pytest.raises(ValueError):
            call()
