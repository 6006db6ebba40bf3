"""Sampling of tokens from shares of their logits: the definition against plain softmax arithmetic, refusals before any launch, and the kernels
against the definition, number by number."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, SSNet, SSNetError, binding
from paper_2406_02629_amd import fixedpoint as fx
from test_adapters import dev, host

gpu = pytest.mark.gpu
ONE = 1 << 30
LOG2E_24 = 2.0 ** 24 / math.log(2)


def weight(distance, scale, h):
    u = distance * scale >> (h + 8)
    octaves, r = u >> 16, u & 0xFFFF
    w = 1077640
    for c in (10033292, 59494488, 257928559, 744260865, 1 << 30):
        w = c - (w * r >> 16)
    return w >> octaves if octaves < 31 else 0


def kept_weights(logits, f, params, allowed=None):
    """logits: whole numbers with f fraction bits -> {token: weight} of those that may be drawn"""
    scale, top_k, top_p, min_p = (int(v) for v in params)
    h = min(f, 16)
    L = {j: max(1 - (1 << 31), min((1 << 31) - 1, int(v) >> (f - h))) for j, v in enumerate(logits) if allowed is None or allowed[j]}
    if not L:
        return {}
    top = max(L.values())
    order = sorted(L, key=lambda j: (-L[j], j))
    if scale <= 0:
        order = order[:1]
    elif top_k > 0:
        order = order[:top_k]
    w = {j: weight(top - L[j], max(scale, 1 << 14), h) for j in order}
    if top_p < ONE:
        need, so_far, few = max(1, -(-max(top_p, 0) * sum(w.values()) // ONE)), 0, []
        for j in order:
            if so_far >= need:
                break
            so_far += w[j]
            few.append(j)
        order = few
    return {j: w[j] for j in sorted(order) if w[j] >= max(1, min(min_p, ONE))}


def draw(weights, random):
    total = sum(weights.values())
    if not total:
        return -1, 0
    target, so_far = (random & (1 << 62) - 1) * total >> 62, 0
    for j, w in weights.items():
        so_far += w
        if so_far > target:
            return j, ((w << 30) + total // 2) // total


def params_of(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    return fx.sampling_parameters(temperature, top_k, top_p, min_p)[0].tolist()


# ------------------------------------------------------------------ the definition

@pytest.mark.parametrize("f", [8, 13, 16, 20])
@pytest.mark.parametrize("temperature", [0.3, 1.0, 2.5])
def test_weights_are_the_softmax(f, temperature):
    """u is cut to 2^-16 octaves (a factor up to 1 + 1.06e-5) and scale rounded (2^-15 of itself at most, here 2^-24: 31 octaves of it 1.3e-6), the polynomial
    is off by 2.2e-7, the distance cut to 2^-16 where f is more (1.53e-5 / temperature of the weight); numerator and sum once each; a
    unit of 2^-30 to a token of the sum, and what 31 octaves cut off is less"""
    rng = np.random.default_rng(f)
    x = np.rint(rng.standard_normal(400) * 3 * 2 ** f).astype(np.int64)
    w = kept_weights(x, f, params_of(temperature))
    z = x / 2.0 ** f / temperature
    want = np.exp(z - z.max())
    want /= want.sum()
    got = np.zeros(400)
    total = sum(w.values())
    for j, v in w.items():
        got[j] = v / total
    cut = 2.0 ** -16 / temperature if f > 16 else 0.0
    assert np.all(np.abs(got - want) <= want * 2 * (1.25e-5 + cut) + 401 * 2.0 ** -30)


def test_cuts_keep_what_they_say():
    f = 13
    x = np.array([0, 5, 5, 5, -3, 9, 9, 2]) * (1 << f)
    assert list(kept_weights(x, f, params_of(top_k=4))) == [1, 2, 5, 6]
    assert list(kept_weights(x, f, params_of(0))) == [5]
    assert list(kept_weights(x, f, params_of(top_p=0.0))) == [5]
    # weights in units of the largest: 2 (1) + 3 e^-4 + e^-7 + e^-9 + e^-12 = 2.0560, of which the first is 0.48638
    assert list(kept_weights(x, f, params_of(top_p=0.486))) == [5] and list(kept_weights(x, f, params_of(top_p=0.487))) == [5, 6]
    # e^-4 = 0.0183 of the largest weight
    assert list(kept_weights(x, f, params_of(min_p=0.0184))) == [5, 6] and list(kept_weights(x, f, params_of(min_p=0.0183))) == [1, 2, 3, 5, 6]
    assert kept_weights(x, f, params_of(), np.zeros(8, bool)) == {} and draw({}, 5) == (-1, 0)
    w = {3: 5, 9: 0, 10: 11}
    assert [draw(w, r << 58)[0] for r in range(16)] == [3] * 5 + [10] * 11 and draw(w, 1 << 62)[0] == 3


def test_parameters():
    t = fx.sampling_parameters([0, 1.0, 0.5], 7, [1.0, 0.9, 0.0], 0.25, rows=3)
    assert t.dtype == torch.int32 and t.tolist() == [[0, 7, ONE, ONE // 4], [round(LOG2E_24), 7, round(0.9 * ONE), ONE // 4], [round(2 * LOG2E_24), 7, 0, ONE // 4]]
    lo, hi = fx.sampling_parameters(1477.0)[0, 0], fx.sampling_parameters(0.0113)[0, 0]
    assert (1 << 14) <= lo and hi > 2 ** 30
    for bad in (dict(temperature=-1.0), dict(temperature=0.001), dict(temperature=2000.0), dict(temperature=1.0, top_p=1.1), dict(temperature=1.0, min_p=-0.1),
                dict(temperature=1.0, top_k=-1), dict(temperature=[1.0, 2.0], rows=3), dict(temperature=float("nan"))):
        with pytest.raises(ValueError):
            fx.sampling_parameters(**bad)


# ------------------------------------------------------------------ refusals (nothing is launched)

def test_refusals_before_any_launch():
    s = SSNet(5, 2, device=None)
    lib, ctx = s.lib, s._ctx
    how = binding._Sampling(64, 64, None, 0)

    def sample(logits=64, ld=100, rows=3, vocab=100, ids=(1, 2, 3), h=how, tokens=64, shown=64):
        return lib.ssnet_sample(ctx, logits, ld, rows, vocab, (C.c_int * 8)(*ids), len(ids), None if h is None else C.byref(h), tokens, shown)

    E = binding.EINVAL
    assert sample() == sample(ld=101) == sample(ids=(5, 1, 3, 2)) == sample(h=binding._Sampling(64, 64, 64, 4)) == binding.EWORKSPACE
    assert [sample(logits=None), sample(ld=99), sample(rows=0), sample(vocab=0), sample(ld=1 << 21, vocab=(1 << 20) + 1), sample(h=None), sample(tokens=None),
            sample(shown=None), sample(h=binding._Sampling(None, 64, None, 0)), sample(h=binding._Sampling(64, None, None, 0)),
            sample(h=binding._Sampling(72, 64, None, 0)), sample(h=binding._Sampling(64, 64, 64, 3)), sample(rows=(1 << 20) + 1)] == [E] * 13
    assert sample(ids=(1, 2)) == binding.ESHARES and sample(ids=(1, 2, 6)) == sample(ids=(1, 2, 2)) == sample(ids=(0, 1, 2)) == binding.EID
    assert lib.ssnet_workspace_bytes_sample(ctx, 0, 5) == lib.ssnet_workspace_bytes_sample(None, 1, 5) == 0 < lib.ssnet_workspace_bytes_sample(ctx, 1, 1)
    x = torch.zeros((5, 3, 10), dtype=torch.int64)
    with pytest.raises(TypeError):
        s.sample(x, [1, 2, 3], torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int64))


@gpu
def test_binding_refuses_shapes():
    ss = SSNet(3, 1)
    x = torch.zeros((3, 4, 70), dtype=torch.int64, device="cuda")
    params, random = fx.sampling_parameters(1.0, rows=4, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    assert ss.sample(x, [1, 2], params, random)[0].tolist() == [0] * 4
    allowed = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    assert ss.sample(x, [1, 2], params, random, allowed=allowed)[0].tolist() == [-1] * 4
    for args, kw in (((x.int(), [1, 2], params, random), {}), ((x[:2], [1, 2], params, random), {}), ((x.transpose(1, 2), [1, 2], params, random), {}),
                     ((x, [1, 2], params[:3], random), {}), ((x, [1, 2], params.long(), random), {}), ((x, [1, 2], params, random.int()), {}),
                     ((x, [1, 2], params, random[:3]), {}), ((x, [1, 2], params, random.cpu()), {}), ((x, [1, 2], params, random), dict(allowed=allowed[:, :2])),
                     ((x, [1, 2], params, random), dict(allowed=allowed[:3])), ((x, [1, 2], params, random), dict(tokens=random.int()))):
        with pytest.raises((TypeError, ValueError)):
            ss.sample(*args, **kw)
    for ids, code in (([1], binding.ESHARES), ([1, 4], binding.EID), ([2, 2], binding.EID)):
        with pytest.raises(SSNetError) as e:
            ss.sample(x, ids, params, random)
        assert e.value.code == code


# ------------------------------------------------------------------ the kernels

def check(ss, values, params, random, allowed=None, ids=None, pad=0):
    """values [rows][vocab]: logits as whole numbers with f fraction bits"""
    rows, vocab = values.shape
    n, t, f, p = ss.n, ss.t, ss.f, ss.p
    ids = list(range(1, t + 2)) if ids is None else ids
    shares = orc.share((values % p).astype(np.uint64), n, t, p, 5, 6)
    wide = torch.full((n, rows, vocab + pad), -3, dtype=torch.int64, device="cuda")
    x = wide[:, :, pad // 2:pad // 2 + vocab]
    x.copy_(dev(shares))
    words = None
    if allowed is not None:
        bits = np.zeros((rows, -(-vocab // 32) * 32 + 32), np.uint64)       # a word more than needed
        bits[:, :vocab] = allowed
        words = (bits.reshape(rows, -1, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)
        words[:, -1] = -1
        words = torch.from_numpy(words).cuda()
    got = ss.sample(x, ids, torch.tensor(params, dtype=torch.int32, device="cuda"), torch.tensor(random, device="cuda"), allowed=words)
    tokens, shown = (v.tolist() for v in got)
    for r in range(rows):
        want = draw(kept_weights(values[r], f, params[r], None if allowed is None else allowed[r]), random[r])
        assert (tokens[r], shown[r]) == want, (r, params[r])


RULES = [params_of(), params_of(0), params_of(0.5, 5), params_of(1.0, 1), params_of(1.0, 50, 0.9), params_of(1.3, 0, 0.95), params_of(0.7, 0, 0.3, 0.05),
         params_of(1.0, 0, 1.0, 0.02), params_of(1.0, 0, 0.0), params_of(1.0, 10 ** 6, 0.99, 0.001), params_of(1477.0, 3, 0.5), params_of(0.0113, 0, 0.9),
         params_of(1.0, 200, 1.0, 1.0), [-5, -3, -1, -7], [1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], [2 ** 31 - 1, 0, 1, 1], params_of(100.0)]


def randoms(rng, rows):
    r = rng.integers(0, 1 << 62, rows).tolist()
    r[:3] = [0, (1 << 62) - 1, -1][:rows]      # (of -1 the lowest 62 bits)
    return r


@gpu
@pytest.mark.parametrize("n,t,p,f", [(3, 1, P61, 13), (5, 2, P61, 20), (7, 3, P61, 8), (3, 1, P45, 12), (8, 3, P45, 16)])
@pytest.mark.parametrize("vocab", [1, 2, 31, 64, 1000, 1025, 4096, 9001])
def test_tokens_match_the_definition(n, t, p, f, vocab):
    rng = np.random.default_rng(vocab + f)
    rows = len(RULES)
    values = np.rint(rng.standard_normal((rows, vocab)) * 3 * 2 ** f).astype(np.int64)
    ss = SSNet(n, t, f=f, seed=1, p=p)
    check(ss, values, RULES, randoms(rng, rows))
    check(ss, values, RULES, randoms(rng, rows), allowed=rng.random((rows, vocab)) < 0.4, ids=list(range(n - t, n + 1)), pad=5)


@gpu
@pytest.mark.parametrize("vocab", [7, 2000, 8200])
def test_equal_logits_masks_and_far_ones(vocab):
    """rows of equal logits, of few different ones, of the farthest that the field and 32 bits hold, of rows whose mask leaves nothing or one token"""
    rng = np.random.default_rng(vocab)
    f, p = 13, P61
    ss = SSNet(3, 1, f=f, seed=1, p=p)
    far = (p - 1) // 2
    kinds = [np.zeros(vocab, np.int64), np.full(vocab, -far), rng.integers(-1, 2, vocab) << f, rng.integers(-2, 1, vocab),
             rng.choice([far, -far, 0, 1 << 31, -(1 << 31), (1 << 31) - 1, 1 << 40, -(1 << 40)], vocab), np.arange(vocab) * 3, -np.arange(vocab) * 50]
    values = np.array([k for k in kinds for _ in RULES])
    params = RULES * len(kinds)
    rows = len(params)
    check(ss, values, params, randoms(rng, rows))
    allowed = rng.random((rows, vocab)) < 0.5
    allowed[1::4] = False
    allowed[2::4] = False
    allowed[2::4, vocab // 2] = True
    check(ss, values, params, randoms(rng, rows), allowed=allowed)


@gpu
@pytest.mark.parametrize("rows,vocab", [(1, 70001), (3, 200003), (12, 33000), (2, 1 << 20)])
@pytest.mark.parametrize("rule", range(0, len(RULES), 4))
def test_large_vocabularies(rows, vocab, rule):
    rng = np.random.default_rng(rows)
    ss = SSNet(3, 1, f=13, seed=1, p=P61)
    values = np.rint(rng.standard_normal((rows, vocab)) * 2 * 2 ** 13).astype(np.int64)
    values[-1, :] >>= 12                        # few different ones
    params = [RULES[(rule + i) % len(RULES)] for i in range(rows)]
    check(ss, values, params, randoms(rng, rows))


@gpu
def test_every_token_is_drawn_as_often_as_its_weight_says():
    """random numbers on a grid of 4096: a token's share of them is its share of the weights up to one at each end"""
    f, vocab, rows = 13, 50, 4096
    rng = np.random.default_rng(1)
    ss = SSNet(3, 1, f=f, seed=1)
    values = np.rint(rng.standard_normal(vocab) * 2 ** f).astype(np.int64)
    shares = orc.share(np.tile(values % P61, (rows, 1)).astype(np.uint64), 3, 1, P61, 5, 6)
    params = fx.sampling_parameters(0.9, 20, 0.97, rows=rows, device="cuda")
    tokens, _ = ss.sample(dev(shares), [1, 2], params, (torch.arange(rows, device="cuda") << 50))
    w = kept_weights(values, f, params[0].tolist())
    count = np.bincount(tokens.cpu().numpy(), minlength=vocab)
    for j in range(vocab):
        assert abs(count[j] - rows * w.get(j, 0) / sum(w.values())) <= 1


@gpu
def test_on_a_stream_of_its_own_and_in_a_graph():
    f, vocab, rows = 13, 40000, 3
    rng = np.random.default_rng(1)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ss = SSNet(3, 1, f=f, seed=1, stream=stream.cuda_stream)
        x = torch.zeros((3, rows, vocab), dtype=torch.int64, device="cuda")
        params, random = fx.sampling_parameters(1.0, rows=rows, device="cuda"), torch.zeros(rows, dtype=torch.int64, device="cuda")
        tokens, shown = ss.sample(x, [1, 2], params, random)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ss.sample(x, [1, 2], params, random, tokens=tokens, shown=shown)
        for turn in range(4):
            values = np.rint(rng.standard_normal((rows, vocab)) * 3 * 2 ** f).astype(np.int64)
            rules, r = [RULES[(turn * 3 + i) % len(RULES)] for i in range(rows)], randoms(rng, rows)
            x.copy_(dev(orc.share((values % P61).astype(np.uint64), 3, 1, P61, 5, 6)))
            params.copy_(torch.tensor(rules, dtype=torch.int32)), random.copy_(torch.tensor(r))
            graph.replay()
            stream.synchronize()
            got = list(zip(tokens.tolist(), shown.tolist()))
            assert got == [draw(kept_weights(values[i], f, rules[i]), r[i]) for i in range(rows)]
            again = ss.sample(x, [1, 2], params, random)
            stream.synchronize()
            assert list(zip(again[0].tolist(), again[1].tolist())) == got
