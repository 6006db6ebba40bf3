"""A decoding loop of several requests on shares: an attention layer with each request's own adapters, a head with adapters, and each request's own
parameters of sampling, against the same loop in plain whole numbers.  Every step opens to what it computes, so the tokens have to be the same."""
import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import Adapters, P45, P61, SSNet
from paper_2406_02629_amd import fixedpoint as fx
from paper_2406_02629_amd.attention import Attention
from test_adapters import i32
from test_attention import fixed_scale
from test_attention_layer import Plain
from test_sampling import draw, kept_weights

gpu = pytest.mark.gpu


class Adapted(Plain):
    """the plain layer with an adapter for each sequence: (a_qkv, b_qkv, a_out, b_out) or None"""

    def token(self, name, x, own):
        f = self.f

        def dense(x, w, a, b):
            y = x @ w
            return y if own is None else y + ((x @ a) >> f) @ b

        y = (dense(x, self.w_qkv, *(own[:2] if own else (0, 0))) >> f).reshape(-1, self.dim)
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
        return dense(o, self.w_out, *(own[2:] if own else (0, 0))) >> f


@gpu
@pytest.mark.parametrize("n,t,p,f,bits,vocab", [(3, 1, P61, 13, 26, 300), (5, 2, P61, 13, 13, 9000), (3, 1, P45, 11, 11, 500)])
def test_decoding_loop_gives_the_plain_tokens(n, t, p, f, bits, vocab):
    rng = np.random.default_rng(vocab)
    width, heads, kv, dim, rank = 32, 2, 1, 16, 5
    qkv = (heads + 2 * kv) * dim
    real = lambda *s: rng.standard_normal(s) / s[0] ** 0.5
    whole = lambda w: np.rint(w * 2 ** f).astype(np.int64)
    w_qkv, w_out, w_head, embed = real(width, qkv), real(heads * dim, width), 4 * real(width, vocab), whole(rng.standard_normal((vocab, width)))
    table = fx.rotary_table(64, fx.rotary_frequencies(dim), f)
    ss = SSNet(n, t, f=f, seed=4, p=p)
    stream = iter(range(10 ** 6, 2 * 10 ** 6))

    def share(v):
        return ss.share(torch.from_numpy(np.ascontiguousarray(v % p)).cuda(), stream_id=next(stream))

    # two adapters of the layer, three of the head; request 2 has none in the layer, request 0 none in the head
    pairs = [[(real(K, rank), real(rank, N)) for _ in range(count)] for K, N, count in ((width, qkv, 2), (heads * dim, width, 2), (width, vocab, 3))]
    sets = []
    for group, (K, N) in zip(pairs, ((width, qkv), (heads * dim, width), (width, vocab))):
        sets.append(Adapters(ss, len(group), K, rank, N))
        for i, (a, b) in enumerate(group):
            sets[-1].load(i, share(whole(a)), share(whole(b)))
    layer_of, head_of = {0: 1, 1: 0, 3: 1}, {1: 2, 2: 0, 3: 2}
    layer = Attention(ss, torch.from_numpy(w_qkv), torch.from_numpy(w_out), heads, kv, table.cuda(), pages=12, page_size=16, weight_bits=bits,
                      adapters_qkv=sets[0], adapters_out=sets[1])
    head = ss.pack_weights_linear(share(whole(w_head)))
    plain = Adapted(w_qkv, w_out, heads, kv, table.numpy(), f, bits, p, "half")
    params = fx.sampling_parameters([0.8, 0.0, 1.2, 1.0], [0, 0, 40, 7], [0.9, 1.0, 1.0, 0.95], [0.0, 0.0, 0.05, 0.0], rows=4, device="cuda")

    tokens = {r: rng.integers(0, vocab, 3 + 2 * r).tolist() for r in range(4)}      # prompts of several lengths
    for step in range(4):
        counts = {r: len(v) for r, v in tokens.items()}
        x = np.concatenate([embed[v] for v in tokens.values()])
        y = layer.forward(share(x), counts, layer_of)
        last = torch.from_numpy(np.cumsum(list(counts.values())) - 1).cuda()
        y = y[:, last].contiguous()
        logits = ss.linear_mod_packed(y, head, vocab)
        logits = ss.adapters_mod(sets[2], y, i32([0, 1, 2, 3, 4]), i32([head_of.get(r, -1) for r in counts]), next(stream), base=logits, out=logits)
        logits = ss.degree_reduce_truncate(logits, next(stream))
        random = torch.from_numpy(rng.integers(0, 1 << 62, 4)).cuda()
        got, shown = ss.sample(logits.view(n, 4, vocab), list(range(n - t, n + 1)), params, random)

        for i, (r, v) in enumerate(tokens.items()):
            own = layer_of.get(r)
            own = None if own is None else [whole(m) for group in pairs[:2] for m in group[own]]
            for token in v:
                z = plain.token(r, embed[token], own)
            full = z @ whole(w_head)
            if r in head_of:
                a, b = (whole(m) for m in pairs[2][head_of[r]])
                full = full + ((z @ a) >> f) @ b
            assert (int(got[i]), int(shown[i])) == draw(kept_weights(full >> f, f, params[i].tolist()), int(random[i])), (step, r)
        tokens = {r: [int(got[i])] for i, r in enumerate(tokens)}


@gpu
def test_a_layer_takes_its_own_adapters_and_stream_ids():
    ss = SSNet(3, 1, f=13, seed=4)
    w_qkv, w_out = torch.zeros((32, 64), dtype=torch.float64), torch.zeros((32, 32), dtype=torch.float64)
    table = fx.rotary_table(64, fx.rotary_frequencies(16), 13).cuda()
    with pytest.raises(ValueError, match="adapters_out"):
        Attention(ss, w_qkv, w_out, 2, 1, table, pages=4, adapters_out=Adapters(ss, 1, 32, 4, 64))
    x = torch.zeros((3, 2, 32), dtype=torch.int64, device="cuda")
    bare = Attention(ss, w_qkv, w_out, 2, 1, table, pages=4, stream_base=1000)
    with pytest.raises(ValueError, match="no adapters"):
        bare.forward(x, {0: 2}, {0: 0})
    assert bare.stream == 1000 and not bare.sequences.length
    bare.forward(x, {0: 2})
    assert bare.stream == 1008
    own = Attention(ss, w_qkv, w_out, 2, 1, table, pages=4, stream_base=2000, adapters_qkv=Adapters(ss, 1, 32, 4, 64))
    own.forward(x, {0: 2}, {0: 0, 5: 7})
    assert own.stream == 2010 and own.sequences.length == {0: 2}
    own.forward(x, {0: 2})
    assert own.stream == 2018
