"""Low-rank adapters of many requests beside a shared projection: refusals before any launch, the layout of a set, and the kernels against the
oracle's products, reduction and truncation, bit for bit."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import Adapters, P45, P61, SSNet, SSNetError, binding

gpu = pytest.mark.gpu
EDGES = lambda p: np.array([0, 1, p - 1, (p - 1) // 2, (p + 1) // 2, 127, 128, 1 << 39], np.uint64)


def uniform(shape, p, rng):
    x = rng.integers(0, p, shape, dtype=np.uint64)
    flat = x.reshape(-1)
    flat[rng.integers(0, flat.size, 8)] = EDGES(p)
    return x


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int64)).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint64)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def reference(x, sets, counts, index, base, n, t, f, p, seed, stream):
    """sets: (a [n][K][r], b [n][r][N]) or None of each place; index: the place of each request"""
    rank = max(s[0].shape[2] for s in sets if s is not None)
    tokens, N = x.shape[1], next(s[1].shape[2] for s in sets if s is not None)
    z2 = np.zeros((n, tokens, rank), np.uint64)
    y = np.zeros((n, tokens, N), np.uint64) if base is None else base.copy()
    places, first = [], 0
    for c, i in zip(counts, index):
        if c and 0 <= i < len(sets) and sets[i] is not None:
            places.append((slice(first, first + c), sets[i]))
        first += c
    for at, (a, _) in places:
        z2[:, at, :a.shape[2]] = orc.linear(x[:, at], a, p)
    z = orc.truncate(orc.degree_reduce(z2.reshape(n, -1), n, t, p, seed, stream), n, t, f, p, seed, stream).reshape(n, tokens, rank)
    for at, (_, b) in places:
        y[:, at] = (y[:, at] + orc.linear(np.ascontiguousarray(z[:, at, :b.shape[1]]), b, p)) % np.uint64(p)
    return y


def make(n, t, p, f, K, N, rank, places, rng, ranks=None):
    sets = []
    for i in range(places):
        r = rank if ranks is None else ranks[i]
        sets.append((uniform((n, K, r), p, rng), uniform((n, r, N), p, rng)) if r else None)
    return sets


def load(ss, sets, K, rank, N):
    s = Adapters(ss, len(sets), K, rank, N)
    for i, ab in enumerate(sets):
        if ab is not None:
            s.load(i, dev(ab[0]), dev(ab[1]))
    return s


# ------------------------------------------------------------------ refusals (nothing is launched)

def test_refusals_before_any_launch():
    s = SSNet(5, 2, device=None)
    lib, ctx = s.lib, s._ctx
    big = 1 << 40
    sets = binding._AdaptersStruct(64, 64, 4, 100, 16, 60)
    reqs = binding._Requests(64, 64, 3, 7)

    def changed(struct, **values):
        new = type(struct).from_buffer_copy(struct)
        for name, value in values.items():
            setattr(new, name, value)
        return new

    def mod(c=sets, r=reqs, x=64, ld_x=100, base=None, ld_base=60, y=big, ld_y=60):
        return lib.ssnet_adapters_mod(ctx, C.byref(c), C.byref(r), x, ld_x, base, ld_base, 0, y, ld_y)

    def pack(c=sets, index=0, a=64, b=64, rank=16):
        return lib.ssnet_pack_adapter(ctx, C.byref(c), index, a, b, rank)

    E = binding.EINVAL
    assert mod() == mod(base=big) == mod(base=big, ld_base=61, ld_y=61) == mod(ld_x=101) == binding.EWORKSPACE
    assert [mod(x=None), mod(y=None), mod(ld_x=99), mod(ld_y=59), mod(base=big, ld_base=59), mod(base=big + 8), mod(base=big, ld_base=61),
            mod(x=big + 8)] == [E] * 8
    for bad in (dict(d_down=None), dict(d_up=None), dict(d_down=72), dict(d_up=72), dict(adapters=0), dict(K=0), dict(K=16384), dict(rank=0),
                dict(rank=129), dict(N=0), dict(N=(1 << 20) + 1), dict(adapters=(1 << 20) + 1)):
        assert mod(c=changed(sets, **bad)) == pack(c=changed(sets, **bad)) == E, bad
    for bad in (dict(d_start=None), dict(d_adapter=None), dict(requests=0), dict(tokens=0), dict(requests=(1 << 20) + 1), dict(tokens=(1 << 24) + 1)):
        assert mod(r=changed(reqs, **bad)) == E, bad
    assert [pack(index=-1), pack(index=4), pack(a=None), pack(b=None), pack(rank=0), pack(rank=17)] == [E] * 6
    # 2t+1 parties, blocks of 64 elements with 64 bytes a limb and rank; n parties, blocks of 32 columns
    assert lib.ssnet_adapter_down_bytes(ctx, 100, 5) == 5 * 2 * 8 * 64 * 5 and lib.ssnet_adapter_up_bytes(ctx, 5, 33) == 5 * 64 * 8 * 8
    other = SSNet(4, 1, p=P45, device=None)
    assert other.lib.ssnet_adapter_down_bytes(other._ctx, 64, 16) == 3 * 6 * 64 * 16 and other.lib.ssnet_adapter_up_bytes(other._ctx, 17, 32) == 4 * 32 * 6 * 32
    assert lib.ssnet_adapter_down_bytes(ctx, 0, 5) == lib.ssnet_adapter_up_bytes(ctx, 129, 5) == lib.ssnet_adapter_down_bytes(None, 1, 1) == 0
    one, many = (lib.ssnet_workspace_bytes_adapters(ctx, C.byref(sets), 1, k) for k in (1, 600))
    assert binding.WS_HEADER_BYTES < one < many and lib.ssnet_workspace_bytes_adapters(ctx, C.byref(sets), 0, 1) == 0
    with pytest.raises(SSNetError):
        Adapters(s, 1, 64, 129, 64)
    with pytest.raises(SSNetError):
        Adapters(s, 0, 64, 16, 64)


class Held:      # what the binding reads of a set, without memory on a GPU
    def __init__(self, ss, K, rank, N):
        self.n, self.t, self.p, self.K, self.rank, self.N = ss.n, ss.t, ss.p, K, rank, N


def test_binding_refuses_other_schemes_and_host_tensors():
    ss = SSNet(5, 2, device=None)
    x, start, index = torch.zeros((5, 3, 16), dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for other in (SSNet(5, 2, p=P45, device=None), SSNet(6, 2, device=None), SSNet(5, 1, device=None)):
        with pytest.raises(ValueError, match="adapters"):
            ss.adapters_mod(Held(other, 16, 4, 16), x, start, index, 0)
    with pytest.raises(TypeError):
        ss.adapters_mod(Held(ss, 16, 4, 16), x, start, index, 0)


@gpu
def test_binding_refuses_shapes():
    ss = SSNet(3, 1)
    s = Adapters(ss, 2, 16, 4, 10)
    x, base = torch.zeros((3, 5, 16), dtype=torch.int64, device="cuda"), torch.zeros((3, 5, 10), dtype=torch.int64, device="cuda")
    start, index = i32([0, 2, 5]), i32([0, 1])
    assert ss.adapters_mod(s, x, start, index, 0).shape == (3, 5, 10)
    for bad in (x[:, :, :15], x[:2], x.transpose(1, 2), x[:, ::2][:, :, ::2], x.int()):
        with pytest.raises((TypeError, ValueError)):
            ss.adapters_mod(s, bad, start, index, 0)
    for kw in (dict(base=base[:, :4]), dict(base=base.int()), dict(out=base[:, :, :9]), dict(base=base.cpu())):
        with pytest.raises((TypeError, ValueError)):
            ss.adapters_mod(s, x, start, index, 0, **kw)
    for bad in ((start[:2], index), (start.long(), index), (start, index.cpu())):
        with pytest.raises((TypeError, ValueError)):
            ss.adapters_mod(s, x, *bad, 0)
    with pytest.raises(SSNetError):
        ss.adapters_mod(s, x, start, index, 0, out=x.view(-1)[:150].view(3, 5, 10))       # the result over the input
    a, b = torch.zeros((3, 16, 4), dtype=torch.int64, device="cuda"), torch.zeros((3, 4, 10), dtype=torch.int64, device="cuda")
    for bad in ((a[:, :15].contiguous(), b), (a, b[:, :3].contiguous()), (a.cpu(), b), (a.int(), b)):
        with pytest.raises((TypeError, ValueError)):
            s.load(0, *bad)
    with pytest.raises(SSNetError):
        s.load(2, a, b)
    with pytest.raises(SSNetError):
        Adapters(ss, 2, 16, 4, 10, down=torch.zeros(5, dtype=torch.int8, device="cuda"))


# ------------------------------------------------------------------ against the oracle

SCHEMES = [(3, 1, P61, 13), (5, 2, P61, 13), (4, 1, P61, 9), (7, 3, P61, 13), (3, 1, P45, 12), (6, 2, P45, 12), (8, 3, P45, 11)]
# (K, N, rank, tokens of the requests, their places)
SHAPES = [
    (1, 1, 1, [1], [0]),                                        # the smallest
    (64, 32, 8, [1], [1]),                                      # one block of everything
    (65, 33, 9, [1, 1, 1, 1, 1], [0, 2, 1, 1, -1]),             # just past a block, single tokens, one without an adapter
    (100, 47, 5, [3, 0, 17, 1, 33], [2, 0, 1, 9, 0]),           # no tokens; a place outside the set
    (130, 70, 16, [16, 16], [0, 0]),                            # whole tiles
    (256, 96, 24, [15, 1, 18], [1, 0, 1]),
    (1000, 130, 32, [2, 2, 2], [0, 1, 2]),                      # two tokens each
    (333, 257, 40, [5, 40], [2, 1]),
    (512, 64, 64, [64], [0]),
    (190, 66, 128, [7, 30, 1], [0, 1, 2]),
    (64, 1030, 16, [21], [1]),                                  # wide
    (3001, 18, 7, [9], [0]),                                    # long
    # single tokens that share adapters: more of one than a tile has, requests beyond a wave's lanes, of no tokens and of several among them
    (64, 130, 12, [1] * 90, [0] * 90),
    (70, 40, 20, [1, 0, 2, 1] * 40, [(7 * i) % 5 - 1 for i in range(160)]),
    (96, 200, 70, [1, 1, 0, 3, 1, 1] * 11, [i % 3 for i in range(66)]),
    (64, 36, 4, [0] * 63 + [1, 1, 5, 1] + [0] * 61 + [1, 4] + [1] * 9, [0] * 128 + [1, 0, 1, 2, 0, 0, 3, 0, 0, 0, 0]),
    (64, 33, 8, [1] * 1030, [i % 4 for i in range(1030)]),
    # so many tiles that each wave of the first product has its own
    (64, 34, 5, [2100, 0, 3, 900, 17], [1, 0, -1, 2, 0]),
    (63, 30, 16, [3001], [2]),
]


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}-{s[1]}-{s[2]}")
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
def test_adapters_match_the_oracle(n, t, p, f, shape):
    K, N, rank, counts, index = shape
    rng = np.random.default_rng(K + N + n)
    sets = make(n, t, p, f, K, N, rank, 3, rng)
    tokens = sum(counts)
    x, base = uniform((n, tokens, K), p, rng), uniform((n, tokens, N), p, rng)
    ss = SSNet(n, t, f=f, seed=11, p=p)
    held = load(ss, sets, K, rank, N)
    start = i32(np.concatenate([[0], np.cumsum(counts)]).tolist())
    want = reference(x, sets, counts, index, base, n, t, f, p, 11, 5)
    assert np.array_equal(host(ss.adapters_mod(held, dev(x), start, i32(index), 5, base=dev(base))), want)


@gpu
@pytest.mark.parametrize("n,t,p,f", [(5, 2, P61, 13), (3, 1, P45, 12)])
@pytest.mark.parametrize("counts", [[1] * 70, [3, 1, 1, 20], [130]])
def test_base_output_and_strides(n, t, p, f, counts):
    """no base, a base in place, parts of longer rows with odd strides, and memory around them that stays"""
    K, N, rank = 96, 80, 16
    rng = np.random.default_rng(8)
    sets = make(n, t, p, f, K, N, rank, 3, rng)
    tokens, index = sum(counts), [(i % 4) - 1 for i in range(len(counts))]
    x, base = uniform((n, tokens, K), p, rng), uniform((n, tokens, N), p, rng)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = load(ss, sets, K, rank, N)
    args = i32(np.concatenate([[0], np.cumsum(counts)]).tolist()), i32(index), 6
    want = reference(x, sets, counts, index, base, n, t, f, p, 3, 6)
    alone = reference(x, sets, counts, index, None, n, t, f, p, 3, 6)
    assert np.array_equal(host(ss.adapters_mod(held, dev(x), *args)), alone)
    inplace = dev(base)
    assert ss.adapters_mod(held, dev(x), *args, base=inplace, out=inplace) is inplace and np.array_equal(host(inplace), want)
    for pad, off in ((7, 3), (6, 2), (16, 0), (5, 0)):
        wide = torch.full((n, tokens, K + pad), -9, dtype=torch.int64, device="cuda")
        wide[:, :, off:off + K] = dev(x)
        for outpad in (pad, 0):
            b, o = (torch.full((n, tokens, N + q), -7, dtype=torch.int64, device="cuda") for q in (pad, outpad))
            bv, ov = b[:, :, off:off + N], o[:, :, min(off, outpad):min(off, outpad) + N]
            bv.copy_(dev(base))
            ss.adapters_mod(held, wide[:, :, off:off + K], *args, base=bv, out=ov)
            assert np.array_equal(host(ov.contiguous()), want)
            assert int((o == -7).sum()) == o.numel() - ov.numel()


@gpu
def test_smaller_ranks_replaced_and_empty_places():
    """adapters of several ranks in one set, a place loaded twice (the second time with a smaller rank), one that was never loaded"""
    n, t, p, f, K, N, rank = 3, 1, P61, 13, 70, 40, 24
    rng = np.random.default_rng(2)
    sets = make(n, t, p, f, K, N, rank, 4, rng, ranks=[24, 3, 17, 0])
    counts, index = [4, 4, 20, 6], [0, 1, 2, 3]
    tokens = sum(counts)
    x, base = uniform((n, tokens, K), p, rng), uniform((n, tokens, N), p, rng)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = load(ss, make(n, t, p, f, K, N, rank, 3, rng) + [None], K, rank, N)
    for i in range(3):
        held.load(i, dev(sets[i][0]), dev(sets[i][1]))
    start = i32(np.concatenate([[0], np.cumsum(counts)]).tolist())
    # a place without an adapter has zeros, whose product still is a sharing: y opens to base there, the shares may differ
    got = host(ss.adapters_mod(held, dev(x), start, i32(index), 5, base=dev(base)))
    padded = [None if s is None else (np.concatenate([s[0], np.zeros((n, K, rank - s[0].shape[2]), np.uint64)], 2),
                                      np.concatenate([s[1], np.zeros((n, rank - s[1].shape[1], N), np.uint64)], 1)) for s in sets]
    assert np.array_equal(got, reference(x, padded, counts, index, base, n, t, f, p, 3, 5))


@gpu
def test_result_opens_to_the_adapted_layer():
    """the sum with the shared projection, reduced and truncated, opens to floor((x W + floor(x A) B) / 2^f) of the encoded values"""
    n, t, p, f, K, N, rank, tokens = 5, 2, P61, 13, 50, 30, 6, 9
    rng = np.random.default_rng(4)
    x, w, a, b = (np.rint(rng.standard_normal(s) * 2 ** f / s[0] ** 0.5).astype(np.int64) for s in ((tokens, K), (K, N), (K, rank), (rank, N)))
    ss = SSNet(n, t, f=f, seed=3, p=p)
    sh = lambda v, i: ss.share(dev((v % p).astype(np.uint64)), i)
    xs = sh(x, 1)
    y = ss.linear_mod_packed(xs, ss.pack_weights_linear(sh(w, 2)), N)
    held = Adapters(ss, 1, K, rank, N)
    held.load(0, sh(a, 3), sh(b, 4))
    y = ss.adapters_mod(held, xs, i32([0, 4, tokens]), i32([0, -1]), 5, base=y, out=y)
    got = orc.lift(host(ss.reconstruct(ss.degree_reduce_truncate(y, 6), [1, 2, 3])), p).reshape(tokens, N)
    change = ((x @ a) >> f) @ b
    change[4:] = 0
    assert np.array_equal(got, (x @ w + change) >> f)


@gpu
def test_tokens_outside_the_requests_stay():
    """a batch padded behind the last request: its rows are not written, and starts beyond the tokens read and write nothing"""
    n, t, p, f, K, N, rank = 3, 1, P61, 13, 64, 48, 8
    rng = np.random.default_rng(2)
    sets = make(n, t, p, f, K, N, rank, 1, rng)
    x, base = uniform((n, 40, K), p, rng), uniform((n, 40, N), p, rng)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = load(ss, sets, K, rank, N)
    want = reference(x, sets, [21, 19], [0, -1], base, n, t, f, p, 3, 5)
    for start, index in (([0, 21], [0]), ([0, 21, 21], [0, 0]), ([-5, 21], [0])):
        out = torch.full((n, 40, N), -7, dtype=torch.int64, device="cuda")
        ss.adapters_mod(held, dev(x), i32(start), i32(index), 5, base=dev(base), out=out)
        assert np.array_equal(host(out[:, :21].contiguous()), want[:, :21]) and bool((out[:, 21:] == -7).all())
    out = torch.full((n, 40, N), -7, dtype=torch.int64, device="cuda")
    ss.adapters_mod(held, dev(x), i32([40, 99]), i32([0]), 5, base=dev(base), out=out)
    assert bool((out == -7).all())


@gpu
def test_a_workspace_that_is_too_small_and_the_messages():
    n, t, p, f, K, N, rank, tokens = 5, 2, P61, 13, 80, 40, 12, 19
    rng = np.random.default_rng(2)
    sets = make(n, t, p, f, K, N, rank, 1, rng)
    x = uniform((n, tokens, K), p, rng)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = load(ss, sets, K, rank, N)
    need = ss.lib.ssnet_workspace_bytes_adapters(ss._ctx, held._address, 1, tokens)
    ss.adapters_mod(held, dev(x), i32([0, tokens]), i32([0]), 5)
    assert ss._ws.numel() == need
    # messages behind the header as ssnet_degree_reduce_truncate leaves them
    count = tokens * rank
    _, msg1, msg2, _ = orc.degree_reduce(orc.linear(x, sets[0][0], p).reshape(n, -1), n, t, p, 3, 5, full=True)
    got = host(ss.messages()[:msg1.size + msg2.size])
    assert np.array_equal(got[:msg1.size], msg1.reshape(-1)) and np.array_equal(got[msg1.size:], msg2.reshape(-1)) and msg1.size == 15 * count
    small = torch.empty(need - 256, dtype=torch.uint8, device="cuda")
    ss._ok(ss.lib.ssnet_set_workspace(ss._ctx, small.data_ptr(), small.numel()), "")
    with pytest.raises(SSNetError) as e:
        ss.adapters_mod(held, dev(x), i32([0, tokens]), i32([0]), 5)
    assert e.value.code == binding.EWORKSPACE


@gpu
def test_on_a_stream_of_its_own_and_in_a_graph():
    n, t, p, f, K, N, rank = 3, 1, P61, 13, 512, 200, 16
    rng = np.random.default_rng(6)
    sets = make(n, t, p, f, K, N, rank, 3, rng)
    counts = [1, 1, 30, 1]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ss = SSNet(n, t, f=f, seed=3, p=p, stream=stream.cuda_stream)
        held = load(ss, sets, K, rank, N)
        x, base, index = (torch.zeros((n, 33, w), dtype=torch.int64, device="cuda") for w in (K, N, 1))
        index = i32([0, 0, 0, 0])
        start = i32([0, 1, 2, 32, 33])
        out = ss.adapters_mod(held, x, start, index, 5, base=base)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ss.adapters_mod(held, x, start, index, 5, base=base, out=out)
        for turn in range(4):
            xv, bv, iv = uniform((n, 33, K), p, rng), uniform((n, 33, N), p, rng), [(turn + i) % 4 - 1 for i in range(4)]
            x.copy_(dev(xv)), base.copy_(dev(bv)), index.copy_(i32(iv))
            graph.replay()
            stream.synchronize()
            got = host(out)
            assert np.array_equal(got, reference(xv, sets, counts, iv, bv, n, t, f, p, 3, 5))
            eager = ss.adapters_mod(held, x, start, index, 5, base=base)
            stream.synchronize()
            assert np.array_equal(host(eager), got)


@gpu
def test_a_pending_product_stays():
    """the product that a dense layer left in the workspace is not touched by adapters in between"""
    n, t, p, f, K, N, rank = 3, 1, P61, 13, 128, 64, 8
    rng = np.random.default_rng(6)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = load(ss, make(n, t, p, f, K, N, rank, 1, rng), K, rank, N)
    xs, packed = ss.share_packed(dev(uniform((16, K), p, rng)), stream_id=1)
    w = ss.pack_weights_linear(dev(uniform((n, K, N), p, rng)))
    ss.reserve(8 << 20)
    ss.linear_product_prepacked(packed, w, 16, K, N)
    want = ss.degree_reduce_truncate(None, 4, out=torch.empty((n, 16 * N), dtype=torch.int64, device="cuda")).clone()
    ss.linear_product_prepacked(packed, w, 16, K, N)
    ss.adapters_mod(held, xs.view(n, 16, K), i32([0, 16]), i32([0]), 5)
    assert torch.equal(ss.degree_reduce_truncate(None, 4, out=torch.empty((n, 16 * N), dtype=torch.int64, device="cuda")), want)
