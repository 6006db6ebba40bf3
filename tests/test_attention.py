"""Rotary positions, the paged cache and attention on shares: the oracle against plain arithmetic, refusals before any launch, and the
kernels against the oracle, bit for bit, at the sizes and masks where they can go wrong."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, PagedCache, SSNet, SSNetError, binding
from paper_2406_02629_amd import fixedpoint as fx

gpu = pytest.mark.gpu


def shares_of(values, n, t, f, p, seed):
    return orc.share(orc.encode(values, f, p), n, t, p, seed, 900 + seed)


def fixed_scale(dim):
    return round(dim ** -0.5 * math.log2(math.e) * (1 << 24))


# ------------------------------------------------------------------ the oracle

@pytest.mark.parametrize("f,scale", [(13, 1 << 24), (13, fixed_scale(128)), (8, fixed_scale(64)), (20, fixed_scale(32))])
def test_weight_of_a_distance_is_a_power_of_two(f, scale):
    """w = 2^30 2^-x up to: x cut to 2^-16 octaves (a factor up to 1 + 1.06e-5), the distance cut to 2^-24 (with the scale at most 2^26: 3e-7),
    the polynomial 2.2e-7, one unit of the shift"""
    rng = np.random.default_rng(3)
    for below in [0, 1, 2, 3] + [int(v) for v in 2 ** rng.uniform(0, 40, 300)]:
        octaves = below / 2.0 ** (2 * f) * scale / 2.0 ** 24
        w = orc.softmax_weight(below, f, scale)
        if octaves >= 31.01:
            assert w == 0
        elif octaves < 30.99:
            assert 2.0 ** (30 - octaves) * (1 - 4e-7) - 1 <= w <= 2.0 ** (30 - octaves) * (1 + 1.2e-5)
    assert orc.softmax_weight(0, f, scale) == 1 << 30


@pytest.mark.parametrize("p", [P61, P45])
@pytest.mark.parametrize("length,bits", [(1, 8), (2, 13), (7, 26), (300, 26), (40000, 30)])
def test_weights_of_a_row_do_not_depend_on_its_mask_and_sum_to_one(p, length, bits):
    rng = np.random.default_rng(length)
    s = (rng.standard_normal(length) * 2 ** 26 * 3).astype(np.int64)
    plain = np.array([orc.softmax_row((s % p).astype(np.uint64), 13, fixed_scale(4), bits, p)])[0]
    for mask in (1, p // 2, p - 5):
        assert np.array_equal(orc.softmax_row(((s + mask % p) % p).astype(np.uint64), 13, fixed_scale(4), bits, p), plain)
    # every weight is rounded to the nearest; before, the sum is 2^bits up to 2^-31 of the reciprocal and 2^-14 of a unit each
    assert abs(int(plain.sum()) - (1 << bits)) <= length * 0.51 + (1 << bits) * 2.0 ** -29
    x = s / 2.0 ** 26 * 0.5
    want = np.exp(x - x.max())
    want /= want.sum()
    # see the test above: 1.2e-5 of a weight, twice (numerator and sum), and what 31 octaves cut off
    assert np.all(np.abs(plain / 2.0 ** bits - want) <= want * 2.6e-5 + 0.51 * 2.0 ** -bits + length * 2.0 ** -30)


def test_digits_of_the_oracle_are_balanced():
    for p, count in ((P61, 8), (P45, 6)):
        x = np.array([0, 1, 127, 128, 255, 256, 32767, 32768, p - 1, p // 2, p // 3], np.uint64)
        d = orc.digits(x, count)
        assert [sum(int(v) << (8 * i) for i, v in enumerate(row)) for row in d] == [int(v) for v in x]


@pytest.mark.parametrize("n,t,p,f,bits", [(3, 1, P61, 13, 26), (5, 2, P61, 13, 13), (3, 1, P45, 10, 10)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_the_oracle_opens_to_softmax_attention(n, t, p, f, bits, causal):
    c, length, heads, kv, dim = 3, 20, 4, 2, 16
    rng = np.random.default_rng(5)
    q, k, v = (np.round(rng.standard_normal(s) * 2 ** f) / 2 ** f for s in ((c, heads, dim), (length, kv, dim), (length, kv, dim)))
    out = orc.attention(*(shares_of(x, n, t, f, p, 1 + i) for i, x in enumerate((q, k, v))), t, f, fixed_scale(dim), bits, causal, p, 9, 4)
    got = orc.decode(orc.reconstruct(out.reshape(n, -1), list(range(1, 2 * t + 2)), p), f + bits, p).reshape(c, heads, dim)
    for i in range(c):
        limit = length - c + i + 1 if causal else length
        for h in range(heads):
            s = k[:limit, h // 2] @ q[i, h] / math.sqrt(dim)
            w = np.exp(s - s.max())
            want = w @ v[:limit, h // 2] / w.sum()
            # weights: see above, and 31 octaves of a scale that is off by 2^-22 of itself (2e-6 each way); keys round to 2^-bits
            assert np.max(np.abs(got[i, h] - want)) <= np.abs(v).max() * (4e-5 + limit * (2.0 ** -bits + 2.0 ** -29))


def test_rotary_of_the_oracle_turns_pairs():
    n, t, f, p, tokens, heads, dim, rot = 3, 1, 16, P61, 4, 2, 12, 8
    x = np.random.default_rng(1).standard_normal((tokens, heads, dim))
    freq = fx.rotary_frequencies(rot)
    table, pos = fx.rotary_table(50, freq, f).numpy(), np.array([0, 3, 49, 7])
    for interleaved in (False, True):
        out = orc.rotary_truncate(shares_of(x, n, t, f, p, 2), table, pos, t, f, p, 5, 6, interleaved)
        got = orc.decode(orc.reconstruct(out.reshape(n, -1), [1, 2], p), f, p).reshape(tokens, heads, dim)
        want = x.copy()
        for a in range(tokens):
            for j in range(rot // 2):
                i0, i1 = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
                z = (x[a, :, i0] + 1j * x[a, :, i1]) * np.exp(1j * pos[a] * freq[j].item())
                want[a, :, i0], want[a, :, i1] = z.real, z.imag
        # the element and the table are rounded to 2^-17, the product cut to 2^-16
        assert np.max(np.abs(got - want)) <= 2.0 ** -16 * (1 + 2 * 0.5 + np.abs(x).max())


# ------------------------------------------------------------------ tables

def test_frequencies_for_longer_contexts():
    plain = fx.rotary_frequencies(64)
    assert plain[0] == 1 and torch.allclose(plain[1:] / plain[:-1], plain[1] / plain[0])
    assert torch.equal(fx.rotary_frequencies(64, factor=4.0), plain / 4)
    parts = fx.rotary_frequencies(64, factor=8.0, original=2048, low=1.0, high=32.0)
    turns = 2048 * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.allclose(parts[turns <= 1], plain[turns <= 1] / 8)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (parts[between] < plain[between]).all() and (parts[between] > plain[between] / 8).all()
    with pytest.raises(ValueError):
        fx.rotary_frequencies(7)
    with pytest.raises(ValueError):
        fx.rotary_table(4, plain, 31, magnitude=1.5)
    assert fx.rotary_table(3, plain, 13).shape == (3, 32, 2) and fx.rotary_table(3, plain, 13)[0, 0].tolist() == [8192, 0]


# ------------------------------------------------------------------ refusals (nothing is launched)

def test_refusals_before_any_launch():
    s = SSNet(5, 2, device=None)
    lib, ctx = s.lib, s._ctx
    rot = binding._Rotary(64, 64, 10, 32, 0)
    cache = binding._PagedCacheStruct(64, 64, 4, 32, 2, 64)
    seqs = binding._Sequences(64, 64, 64, 2, 6, 3, 90)
    addr = C.byref

    def rotary(d_x=64, ld=128, tokens=3, heads=2, dim=64, r=rot, out=1 << 20):
        return lib.ssnet_rotary_truncate(ctx, d_x, ld, tokens, heads, dim, None if r is None else addr(r), 0, out)

    def append(c=cache, k=64, ld=128, tokens=3, slots=64, r=rot):
        return lib.ssnet_cache_append(ctx, addr(c), k, ld, 64, ld, tokens, slots, None if r is None else addr(r), 0)

    def attend(c=cache, q=64, ld=256, heads=4, scale=1 << 20, bits=13, out=1 << 20, s=seqs):
        return lib.ssnet_paged_attention(ctx, addr(c), addr(s), q, ld, heads, scale, bits, 1, 0, out)

    def changed(struct, **values):
        new = type(struct).from_buffer_copy(struct)
        for name, value in values.items():
            setattr(new, name, value)
        return new

    # right arguments reach the check of the workspace, which is missing
    assert rotary() == append() == attend() == binding.EWORKSPACE
    E = binding.EINVAL
    assert [rotary(d_x=None), rotary(ld=127), rotary(tokens=0), rotary(heads=0), rotary(r=None), rotary(out=None)] == [E] * 6
    assert rotary(tokens=1 << 20, heads=1 << 10) == E                                # more than 2^31 elements
    assert rotary(out=64) == binding.EWORKSPACE and rotary(out=64, ld=129) == E == rotary(out=72)   # in place, or no overlap
    for bad in (dict(d_table=None), dict(d_pos=None), dict(positions=0), dict(rot=0), dict(rot=31), dict(rot=66), dict(d_table=68)):
        assert rotary(r=changed(rot, **bad)) == append(r=changed(rot, **bad)) == E, bad
    for bad in (dict(page_size=0), dict(page_size=24), dict(heads=0), dict(head_dim=0), dict(head_dim=40), dict(head_dim=272), dict(pages=0),
                dict(d_keys=None), dict(d_values=72), dict(pages=1 << 27)):
        assert append(c=changed(cache, **bad)) == attend(c=changed(cache, **bad)) == E, bad
    assert [append(k=None), append(ld=100), append(tokens=0), append(slots=None)] == [E] * 4
    assert [attend(q=None), attend(ld=255), attend(heads=3), attend(heads=0), attend(scale=(1 << 16) - 1), attend(scale=1 << 26),
            attend(bits=7), attend(bits=31), attend(out=None), attend(out=64)] == [E] * 10
    for bad in (dict(d_start=None), dict(d_table=None), dict(d_length=None), dict(sequences=0), dict(tokens=0), dict(max_pages=0),
                dict(max_length=0), dict(max_length=(1 << 20) + 1)):
        assert attend(s=changed(seqs, **bad)) == E, bad
    assert lib.ssnet_cache_page_bytes(ctx, 32, 2, 64) == 5 * 2 * 32 * 64 * 8
    assert lib.ssnet_cache_page_bytes(ctx, 32, 2, 60) == 0 == lib.ssnet_cache_page_bytes(None, 32, 2, 64)
    assert SSNet(3, 1, p=P45, device=None).lib.ssnet_cache_page_bytes(SSNet(3, 1, p=P45, device=None)._ctx, 16, 1, 16) == 3 * 16 * 16 * 6
    one, many = (lib.ssnet_workspace_bytes_attention(ctx, addr(cache), 2, k, 4, 90) for k in (1, 6))
    assert binding.WS_HEADER_BYTES < one < many and lib.ssnet_workspace_bytes_attention(ctx, addr(cache), 2, 6, 3, 90) == 0
    # without a rotation nothing needs the workspace, but a cache on the host is refused by the binding
    with pytest.raises(TypeError):
        PagedCache(s, 2, 32, 2, 64, keys=torch.zeros(2 * 5 * 2 * 32 * 64 * 8, dtype=torch.int8), values=torch.zeros(1, dtype=torch.int8))
    with pytest.raises(SSNetError):
        PagedCache(s, 2, 30, 2, 64)
    x = torch.zeros((5, 3, 2, 64), dtype=torch.int64)
    with pytest.raises(TypeError):
        s.rotary_truncate(x, torch.zeros((4, 16, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 0)


# ------------------------------------------------------------------ the kernels

def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint64).view(np.int64)).to("cuda:0")


def host(t):
    return t.detach().cpu().contiguous().numpy().view(np.uint64)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda:0")


SCHEMES = [(3, 1, P61, 13), (5, 2, P61, 13), (4, 1, P61, 8), (6, 2, P61, 13), (7, 3, P61, 13), (8, 3, P45, 12), (3, 1, P45, 12), (5, 2, P45, 12)]


@gpu
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
@pytest.mark.parametrize("tokens,heads,dim,rot", [(1, 1, 2, 2), (3, 2, 32, 32), (5, 3, 20, 6), (65, 2, 128, 64)])
def test_rotary_matches_the_oracle(n, t, p, f, tokens, heads, dim, rot):
    rng = np.random.default_rng(tokens)
    x = shares_of(rng.standard_normal((tokens, heads, dim)) * 4, n, t, f, p, 3)
    table, pos = fx.rotary_table(200, fx.rotary_frequencies(rot), f).numpy(), rng.integers(0, 200, tokens)
    table[0, 0] = (-(1 << 24), (1 << 24) - 1)         # entries need not be a rotation
    ss = SSNet(n, t, f=f, seed=21, p=p)
    for layout in ("half", "interleaved"):
        want, u, wsh = orc.rotary_truncate(x, table, pos, t, f, p, 21, 5, layout == "interleaved", full=True)
        got = ss.rotary_truncate(dev(x), torch.from_numpy(table).cuda(), i32(pos.tolist()), 5, layout=layout)
        assert np.array_equal(host(got), want)
        count = tokens * heads * rot
        msgs = host(ss.messages())[:(t + 1 + n) * count]
        assert np.array_equal(msgs, np.concatenate([u.reshape(-1), wsh.reshape(-1)]))
        # in place, and from a part of a longer row per token
        d = dev(x)
        assert ss.rotary_truncate(d, torch.from_numpy(table).cuda(), i32(pos.tolist()), 5, layout=layout, out=d) is d
        assert np.array_equal(host(d), want)
        wide = torch.full((n, tokens, heads * dim + 7), -1, dtype=torch.int64, device="cuda")
        part = wide[:, :, 3:3 + heads * dim].unflatten(-1, (heads, dim))
        part.copy_(dev(x))
        assert np.array_equal(host(ss.rotary_truncate(part, torch.from_numpy(table).cuda(), i32(pos.tolist()), 5, layout=layout)), want)


@gpu
def test_rotary_of_field_elements_of_any_size():
    """turned elements of any residue, entries of the table at the ends of 32 bits: the messages of step 1 are the turned shares plus the mask's
    whatever the value is (p/2 bounds only what the truncation means)"""
    for p in (P61, P45):
        n, t, f, tokens, heads, dim = 3, 1, 13, 7, 2, 16
        rng = np.random.default_rng(8)
        x = rng.integers(0, p, (n, tokens, heads, dim), dtype=np.uint64)
        x[:, 0], x[:, 1], x[0, 2], x[1, 2] = p - 1, 0, p - 1, 0
        table = rng.integers(-(1 << 31), 1 << 31, (4, 8, 2)).astype(np.int32)
        table[0] = -(1 << 31)
        table[1] = (1 << 31) - 1
        table[2, :, 0], table[2, :, 1] = -(1 << 31), (1 << 31) - 1
        pos = np.array([0, 1, 2, 2, 0, 1, 3])
        want, u, wsh = orc.rotary_truncate(x, table, pos, t, f, p, 1, 2, full=True)
        ss = SSNet(n, t, f=f, seed=1, p=p)
        got = ss.rotary_truncate(dev(x), torch.from_numpy(table).cuda(), i32(pos.tolist()), 2)
        assert np.array_equal(host(got), want) and np.array_equal(host(ss.messages())[:u.size], u.reshape(-1))


def cells_of(shares, digits, values):
    """[n, places, heads, dim], places a multiple of 16 -> [n, heads, places / 16, digits, ...] int8 as the cache has it"""
    n, places, heads, dim = shares.shape
    d = orc.digits(shares, digits)                                                     # n, place, head, element, digit
    if values:
        return d.reshape(n, places // 16, 16, heads, dim, digits).transpose(0, 3, 1, 5, 4, 2)
    return d.reshape(n, places // 16, 16, heads, dim // 16, 16, digits).transpose(0, 3, 1, 6, 4, 2, 5)


@gpu
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
@pytest.mark.parametrize("tokens,heads,dim,rot,page", [(1, 1, 16, 0, 16), (5, 2, 48, 32, 32), (70, 3, 64, 64, 16), (150, 1, 128, 128, 64), (33, 2, 80, 20, 48),
                                                       (66, 1, 96, 0, 16), (430, 2, 160, 160, 32), (300, 7, 64, 24, 64), (1030, 1, 128, 0, 16),
                                                       (515, 2, 128, 20, 16)])
def test_append_matches_the_oracle(n, t, p, f, tokens, heads, dim, rot, page):
    rng = np.random.default_rng(dim)
    digits = 6 if p == P45 else 8
    k, v = (shares_of(rng.standard_normal((tokens, heads, dim)), n, t, f, p, s) for s in (3, 4))
    pages = -(-tokens // page) + 2
    for order in ("cells", "run", "scattered"):
        slots = np.arange(tokens) + (page // 2 + 5 if order == "run" else 0)
        if order == "scattered":
            slots = rng.permutation(pages * page)[:tokens]
        if tokens > 4:                                      # left out
            slots[1], slots[3] = -1, pages * page
        ss = SSNet(n, t, f=f, seed=21, p=p)
        cache = PagedCache(ss, pages, page, heads, dim)
        cache.keys.random_(-128, 128), cache.values.random_(-128, 128)
        want_k, want_v = cache.keys.cpu().numpy().copy(), cache.values.cpu().numpy().copy()
        turned, kw = k, {}
        if rot:
            table, pos = fx.rotary_table(100, fx.rotary_frequencies(rot), f).numpy(), rng.integers(0, 100, tokens)
            turned = orc.rotary_truncate(k, table, pos, t, f, p, 21, 5, True)
            kw = dict(table=torch.from_numpy(table).cuda(), pos=i32(pos.tolist()), layout="interleaved")
        wide = torch.zeros((n, tokens, heads * dim + 5), dtype=torch.int64, device="cuda")
        wide[:, :, :heads * dim] = dev(v).flatten(2)
        ss.cache_append(cache, dev(k), wide[:, :, :heads * dim].unflatten(-1, (heads, dim)), torch.from_numpy(slots).cuda(), 5, **kw)
        for a, s in enumerate(slots):
            if 0 <= s < pages * page:
                for shares, want, values in ((turned, want_k, False), (v, want_v, True)):
                    cell = np.zeros((n, 16, heads, dim), np.uint64)
                    cell[:, s % 16] = shares[:, a]
                    c = cells_of(cell, digits, values)[:, :, 0]
                    if values:
                        want[s // page, :, :, s % page // 16, :, :, s % 16] = c[..., s % 16]
                    else:
                        want[s // page, :, :, s % page // 16, :, :, s % 16] = c[:, :, :, :, s % 16]
        assert np.array_equal(cache.keys.cpu().numpy(), want_k) and np.array_equal(cache.values.cpu().numpy(), want_v), order


class Context:
    """queries, keys and values of several sequences, a cache that holds them in pages of any order, and the oracle's result"""

    def __init__(self, n, t, p, f, chunks, lengths, heads, kv, dim, page, seed=1, spread=1.0, extra=0):
        rng = np.random.default_rng(seed)
        self.n, self.t, self.p, self.f, self.heads, self.kv, self.dim, self.page = n, t, p, f, heads, kv, dim, page
        self.chunks, self.lengths = chunks, lengths
        self.q = [shares_of(rng.standard_normal((c, heads, dim)) * spread, n, t, f, p, 10 + i) for i, c in enumerate(chunks)]
        self.k = [shares_of(rng.standard_normal((x, kv, dim)) * spread, n, t, f, p, 30 + i) for i, x in enumerate(lengths)]
        self.v = [shares_of(rng.standard_normal((x, kv, dim)), n, t, f, p, 50 + i) for i, x in enumerate(lengths)]
        blocks = [-(-x // page) for x in lengths]
        self.ss = ss = SSNet(n, t, f=f, seed=21, p=p)
        pages = sum(blocks) + 1 + extra
        self.cache = PagedCache(ss, pages, page, kv, dim)
        self.cache.keys.random_(-128, 128), self.cache.values.random_(-128, 128)          # what pages held before
        order, first = rng.permutation(pages), 0
        table = np.full((len(lengths), max(max(blocks), 1)), -7, np.int32)
        for b, count in enumerate(blocks):
            table[b, :count] = order[first:first + count]
            first += count
            if lengths[b]:
                pad = np.zeros((n, count * page - lengths[b], kv, dim), np.uint64)
                for tensor, shares, values in ((self.cache.keys, self.k[b], False), (self.cache.values, self.v[b], True)):
                    c = cells_of(np.concatenate([shares, pad], 1), self.cache.digits, values)
                    whole = c.reshape(c.shape[:2] + (count, page // 16) + c.shape[3:])
                    at = torch.from_numpy(table[b, :count].astype(np.int64)).cuda()
                    new = torch.from_numpy(np.ascontiguousarray(np.moveaxis(whole, 2, 0))).cuda()
                    last = lengths[b] - (count - 1) * page
                    tensor[at[:-1]] = new[:-1]
                    whole_cells = last // 16
                    tensor[at[-1], :, :, :whole_cells] = new[-1, :, :, :whole_cells]
                    if last % 16:                                                          # unused places keep what they held
                        (tensor[at[-1], :, :, whole_cells, ..., :last % 16] if values else tensor[at[-1], :, :, whole_cells, :, :, :last % 16]).copy_(
                            new[-1, :, :, whole_cells, ..., :last % 16] if values else new[-1, :, :, whole_cells, :, :, :last % 16])
        self.table = torch.from_numpy(table).cuda()
        self.start = i32([sum(chunks[:i]) for i in range(len(chunks) + 1)])
        self.ctx = i32(lengths)
        self.queries = dev(np.concatenate(self.q, 1))

    def run(self, bits, causal=True, stream=5, max_ctx=None, q=None, **kw):
        return self.ss.paged_attention(self.cache, self.queries if q is None else q, self.start, self.table, self.ctx,
                                       max(self.lengths + [1]) if max_ctx is None else max_ctx, stream, weight_bits=bits, causal=causal, **kw)

    def want(self, bits, causal=True, stream=5, full=False):
        parts, at = [], 0
        for b, c in enumerate(self.chunks):
            if c:
                parts.append(orc.attention(self.q[b], self.k[b], self.v[b], self.t, self.f, fixed_scale(self.dim), bits, causal, self.p, 21, stream, at, full))
            at += c
        return parts if full else np.concatenate(parts, 1)


@gpu
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_matches_the_oracle_in_every_scheme(n, t, p, f, causal):
    bits = f if p == P45 else 2 * f
    c = Context(n, t, p, f, [2, 1, 5], [40, 1, 18], 4, 2, 32, 16)
    assert np.array_equal(host(c.run(bits, causal)), c.want(bits, causal))


@gpu
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 256])
@pytest.mark.parametrize("heads,kv,page", [(1, 1, 16), (3, 3, 48), (6, 2, 32), (8, 1, 64)])
def test_attention_matches_the_oracle_in_every_head_layout(dim, heads, kv, page):
    c = Context(3, 1, P61, 13, [7, 1], [23, 70], heads, kv, dim, page)
    assert np.array_equal(host(c.run(13)), c.want(13))


@gpu
@pytest.mark.parametrize("lengths", [1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 511, 513, 1025])
@pytest.mark.parametrize("chunk", [1, 3, 40])
def test_attention_at_the_edges_of_tiles(lengths, chunk):
    """contexts around the blocks of 16, 64 and 256 keys, chunks of one tile of rows and of several (40 tokens of 3 heads: 120 rows); the chunk
    may be longer than the context: its first tokens then see nothing and give zero"""
    c = Context(3, 1, P61, 13, [chunk], [lengths], 3, 1, 16, 16)
    got = host(c.run(20))
    assert np.array_equal(got, c.want(20))
    if chunk > lengths:
        assert not got[:, :chunk - lengths].any()


@gpu
def test_sequences_without_tokens_and_without_context():
    c = Context(5, 2, P61, 13, [0, 3, 0, 2, 1, 0], [9, 0, 0, 5, 33, 1], 2, 1, 32, 16)
    for causal in (True, False):
        got = host(c.run(13, causal))
        assert np.array_equal(got, c.want(13, causal)) and not got[:, :3].any()


@gpu
@pytest.mark.parametrize("p,f", [(P61, 13), (P45, 10)])
def test_many_sequences(p, f):
    """more sequences than lanes of a wave, of all lengths"""
    rng = np.random.default_rng(2)
    chunks = [int(v) for v in rng.integers(0, 4, 150)]
    lengths = [int(v) for v in rng.integers(0, 40, 150)]
    c = Context(3, 1, p, f, chunks, lengths, 2, 2, 16, 16)
    assert np.array_equal(host(c.run(f)), c.want(f))


@gpu
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
@pytest.mark.parametrize("chunk,length", [(2, 3000), (300, 1100), (1, 4097), (40, 4500)])
def test_rows_of_every_length_class(n, t, p, f, chunk, length):
    """the softmax of a row in one workgroup, small or large, or in several"""
    c = Context(n, t, p, f, [chunk], [length], 4 if chunk < 100 else 5, 1, 16, 64)
    if chunk == 300:                               # more rows than the oracle need see: its last tokens
        c.q[0] = c.q[0][:, -3:]
        want = orc.attention(c.q[0], c.k[0], c.v[0], t, f, fixed_scale(16), f, True, p, 21, 5, chunk - 3)
        assert np.array_equal(host(c.run(f))[:, -3:], want)
    else:
        assert np.array_equal(host(c.run(f)), c.want(f))


@gpu
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
@pytest.mark.parametrize("chunk,length", [(250, 900), (300, 1100), (700, 2000)])
def test_every_row_of_more_rows_than_the_card_holds_workgroups(n, t, p, f, chunk, length):
    """rows of a chunk whose workgroups follow others on their CU, several calls"""
    c = Context(n, t, p, f, [chunk], [length], 8, 1, 16, 64)
    c.q[0] = c.q[0][:, chunk // 2:]
    want = orc.attention(c.q[0], c.k[0], c.v[0], t, f, fixed_scale(16), f, True, p, 21, 5, chunk - chunk // 2)
    first = c.run(f)
    assert np.array_equal(host(first)[:, chunk // 2:], want)
    for _ in range(3):
        assert torch.equal(c.run(f), first)


@gpu
@pytest.mark.parametrize("n,t", [(3, 1), (5, 2)])
def test_a_long_context_is_joined_from_several_runs(n, t):
    """longer than the 16383 products that a 32-bit sum of digits can take"""
    c = Context(n, t, P61, 13, [2], [17000], 2, 1, 16, 64)
    assert np.array_equal(host(c.run(26)), c.want(26))


@gpu
def test_sharp_and_flat_rows():
    """scores far apart (weights of 0 and 1) and all equal"""
    c = Context(3, 1, P61, 13, [3], [300], 2, 1, 64, 16, spread=30.0)
    assert np.array_equal(host(c.run(26)), c.want(26))
    c = Context(3, 1, P61, 13, [3], [300], 2, 1, 64, 16, spread=0.0)
    want, _, _, weight = c.want(26, full=True)[0]
    assert len(set(weight[0, 0, :298].tolist())) == 1 and np.array_equal(host(c.run(26)), want)


@gpu
@pytest.mark.parametrize("p,bits", [(P61, 8), (P61, 30), (P45, 8)])
def test_weight_bits(p, bits):
    c = Context(3, 1, p, 10, [4], [90], 2, 1, 32, 16)
    assert np.array_equal(host(c.run(bits)), c.want(bits))


@gpu
@pytest.mark.parametrize("f", [1, 5, 20])
def test_fraction_bits(f):
    c = Context(3, 1, P61, f, [4], [90], 2, 1, 32, 16)
    assert np.array_equal(host(c.run(12)), c.want(12))


@gpu
def test_messages_are_the_masked_scores():
    c = Context(5, 2, P61, 13, [3], [70], 2, 1, 32, 16)
    c.run(13)
    _, msg, _, _ = c.want(13, full=True)[0]
    rows, keys = 3 * 2, 128
    m = host(c.ss.messages())[:5 * rows * keys].reshape(5, 3, 2, keys)
    for i in range(3):
        limit = 70 - 3 + i + 1
        assert np.array_equal(m[:, i, :, :limit], msg[:, i, :, :limit])


@gpu
@pytest.mark.parametrize("n,t,p,f", [(5, 2, P61, 13), (3, 1, P45, 12)])
def test_a_small_workspace_gives_the_same_result(n, t, p, f):
    """tokens in several runs, tables wider and bounds longer than needed, a query that is part of a longer row, another memory for the result"""
    c = Context(n, t, p, f, [9, 1, 30], [40, 11, 200], 4, 2, 64, 32, extra=3)
    want = c.want(f)
    assert np.array_equal(host(c.run(f)), want)
    small = SSNet(n, t, f=f, seed=21, p=p)
    small.ATTENTION_ROOM = 0
    c.ss = small
    assert np.array_equal(host(c.run(f)), want)
    assert small._ws.numel() == small.workspace_bytes_attention(c.cache, 3, 1, 4, 200)
    wide = torch.zeros((n, 40, 4 * 64 + 16), dtype=torch.int64, device="cuda")
    wide[:, :, 16:] = c.queries.flatten(2)
    c.table = torch.cat([c.table, torch.full((3, 9), 1 << 30, dtype=torch.int32, device="cuda")], 1).contiguous()
    out = torch.empty((n, 40, 4, 64), dtype=torch.int64, device="cuda")
    assert c.run(f, max_ctx=431, q=wide[:, :, 16:].unflatten(-1, (4, 64)), out=out) is out
    assert np.array_equal(host(out), want)


@pytest.mark.parametrize("tokens,heads,dim,keys", [(1024, 32, 64, 16384), (8192, 8, 128, 8192), (4096, 64, 32, 4000), (100, 8, 64, 1000)])
def test_no_launch_has_2_32_threads(tokens, heads, dim, keys):
    """single tokens of many sequences: the workspace asked for is that of a run of tokens whose workgroups of scores, one of 256 threads to a token, head
    of the cache, party and 128 keys, are fewer (more would be cut off without an error).  It holds the messages and the weights; sums of
    runs of keys add less than 2 % here."""
    for n, t, f, p, digits in ((5, 2, 13, P61, 8), (3, 1, 12, P45, 6), (8, 3, 13, P61, 8)):
        ss = SSNet(n, t, f=f, seed=1, p=p, device=None)
        cache = binding._PagedCacheStruct(None, None, 1, 16, heads, dim)
        need = ss.lib.ssnet_workspace_bytes_attention(ss._ctx, C.addressof(cache), tokens, tokens, heads, keys)
        parties, padded = 2 * t + 1, (keys + 63) // 64 * 64
        run = need / (heads * padded * (8 * parties + digits * n))
        assert run * heads * parties * math.ceil(padded / 128) < 1.02 * 2 ** 24
        if tokens * heads * parties * math.ceil(padded / 128) < 2 ** 24:
            assert run >= tokens


@gpu
@pytest.mark.parametrize("chunks,lengths,heads,kv,dim", [([5, 130], [40, 2600], 48, 1, 64), ([60], [200], 16, 16, 32), ([33], [4500], 20, 1, 96)])
def test_room_for_one_token_serves_a_chunk(chunks, lengths, heads, kv, dim):
    """a chunk whose tokens one by one go other ways than together: larger tiles, fewer runs, softmax and values apart"""
    n, t, f = 5, 2, 13
    c = Context(n, t, P61, f, chunks, lengths, heads, kv, dim, 32)
    want = c.run(f)
    c.ss = SSNet(n, t, f=f, seed=21, p=P61)
    c.ss.ATTENTION_ROOM = 0
    assert torch.equal(c.run(f), want)
    assert c.ss._ws.numel() == c.ss.workspace_bytes_attention(c.cache, len(chunks), 1, heads, max(lengths))


@gpu
def test_workspace_too_small_is_refused_and_a_pending_product_survives():
    n, t = 5, 2
    c = Context(n, t, P61, 13, [2], [70], 2, 1, 32, 16)
    ss = c.ss
    need = ss.workspace_bytes_attention(c.cache, 1, 2, 2, 70)
    room = torch.empty(need + (1 << 20), dtype=torch.uint8, device="cuda")
    seqs = binding._Sequences(c.start.data_ptr(), c.table.data_ptr(), c.ctx.data_ptr(), 1, 2, c.table.shape[1], 70)
    out = torch.zeros((n, 2, 2, 32), dtype=torch.int64, device="cuda")

    def call():
        return ss.lib.ssnet_paged_attention(ss._ctx, c.cache._address, C.byref(seqs), c.queries.data_ptr(), 64, 2, fixed_scale(32), 13, 1, 5, out.data_ptr())

    one = ss.workspace_bytes_attention(c.cache, 1, 1, 2, 70)
    assert ss.lib.ssnet_set_workspace(ss._ctx, room.data_ptr(), one - 256) == 0 and call() == binding.EWORKSPACE
    torch.cuda.synchronize()
    assert not out.any()
    assert ss.lib.ssnet_set_workspace(ss._ctx, room.data_ptr(), room.numel()) == 0
    x, w = (shares_of(np.random.default_rng(s).standard_normal(shape), n, t, 13, P61, s) for s, shape in ((6, (4, 40)), (7, (40, 8))))
    xs, wp = torch.empty(n * ss.lib.ssnet_packed_weight_bytes(4, 40), dtype=torch.uint8, device="cuda"), ss.pack_weights_linear(dev(w))
    assert ss.lib.ssnet_pack_weights_linear(ss._ctx, dev(np.ascontiguousarray(x.transpose(0, 2, 1))).data_ptr(), 40, 4, xs.data_ptr()) == 0
    assert ss.lib.ssnet_linear_product_prepacked(ss._ctx, xs.data_ptr(), wp.data_ptr(), 4, 40, 8) == 0
    assert call() == 0 and np.array_equal(host(out), c.want(13))
    red = torch.empty((n, 32), dtype=torch.int64, device="cuda")
    assert ss.lib.ssnet_degree_reduce(ss._ctx, None, 32, 3, red.data_ptr()) == 0
    assert np.array_equal(host(red), orc.degree_reduce(orc.linear(x, w, P61).reshape(n, -1), n, t, P61, 21, 3))


@gpu
def test_on_a_stream_of_its_own_and_in_a_graph():
    c = Context(3, 1, P61, 13, [3, 1], [100, 60], 4, 2, 64, 16)
    want = c.want(13)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    ss = SSNet(3, 1, f=13, seed=21, stream=stream.cuda_stream)
    c.ss = ss
    with torch.cuda.stream(stream):
        out = c.run(13)
    stream.synchronize()
    assert np.array_equal(host(out), want)
    graph = torch.cuda.CUDAGraph()
    out.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        c.run(13, out=out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(out), want)
        assert int(c.queries.sum()) is not None
