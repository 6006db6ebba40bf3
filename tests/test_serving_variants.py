"""Variants of the kernels of adapter_kernels.hip and sample_kernels.hip that are chosen by sizes and alignment: tensors that go past the caches, element by
element and in pairs.  Which sizes take which variant is checked on the CPU, so that a rule that changes does not leave a variant without its test."""
import ctypes as C
import subprocess

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, SSNet
from paper_2406_02629_amd import fixedpoint as fx
from test_adapters import EDGES, SHAPES, dev, host, i32, load, make, reference, uniform
from test_sampling import draw, kept_weights
from test_serving_sizes import CSRC, AdapterPlan, SamplePlan

gpu = pytest.mark.gpu
SCHEMES = {P61: (3, 1, 13), P45: (3, 1, 12)}     # n, t, f

# (K, N, rank, tokens of the requests, their places): odd lengths of the contraction and odd widths at the ranks that have kernels of their own
ODD = [
    (333, 45, 24, [5, 40], [2, 1]),
    (191, 67, 100, [7, 30, 1], [0, 1, 2]),
]
# second products of more than 256 MB: a long prompt beside single tokens, with and without an adapter; many requests of two tokens that share adapters
PROMPT, PAIRS_OF_TOKENS = ([1999, 0, 1, 100], [0, 1, -1, 2]), ([2] * 1024, [(7 * i) % 4 - 1 for i in range(1024)])
STREAMED = [(64, 2700, 8, *PROMPT), (64, 2700, 16, *PROMPT), (64, 2700, 32, *PROMPT), (64, 2700, 40, *PROMPT),
            (70, 2802, 16, *PAIRS_OF_TOKENS), (70, 2802, 40, *PAIRS_OF_TOKENS)]
# (rows, vocabulary, parties that open): of test_sampling.py and test_serving_sizes.py some, and rows of an even vocabulary that are read past the caches
SAMPLED = [(17, 1000, 2), (17, 9001, 2), (12, 33000, 2), (256, 32768, 2), (2000, 100001, 2)]
SAMPLED_STREAMED = (100, 200000, 2)


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d, libs = tmp_path_factory.mktemp("serving_variants"), {}
    src = d / "serving_variants.cpp"
    src.write_text('#include "serving_plan.hpp"\nextern "C" {\n'
                   "SS_NS::adapter_plan adapters(int n, int t, int tokens, int requests, int K, int rank, int N)\n"
                   "{ return SS_NS::plan_adapters(n, t, tokens, requests, K, rank, N); }\n"
                   "SS_NS::sample_plan sample(int rows, int vocab, size_t room) { return SS_NS::plan_sample(rows, vocab, room); }\n"
                   "size_t steps(size_t rank) { return SS_NS::up_steps(rank); }\n"
                   "size_t streamed() { return SS_NS::STREAMED_BYTES; }\n}\n")
    for p, limbs in ((P61, 8), (P45, 6)):
        so = str(d / f"serving_variants{limbs}.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-DSS_NLIMB={limbs}", "-DSS_NS=rules", "-I", CSRC, "-o", so,
                        str(src)], check=True)
        lib = libs[p] = C.CDLL(so)
        lib.adapters.restype, lib.adapters.argtypes = AdapterPlan, [C.c_int] * 7
        lib.sample.restype, lib.sample.argtypes = SamplePlan, [C.c_int, C.c_int, C.c_size_t]
        lib.steps.restype, lib.steps.argtypes = C.c_size_t, [C.c_size_t]
        lib.streamed.restype = C.c_size_t
    return libs


def test_every_variant_of_the_adapters_has_a_shape(rules):
    """as ss_launch_adapters_down and ss_launch_adapters_up choose them for tensors without gaps"""
    for p, (n, t, _) in SCHEMES.items():
        down, up, streamed = set(), set(), set()
        for shape in SHAPES + ODD + STREAMED:
            K, N, rank, counts, _ = shape
            plan = rules[p].adapters(n, t, sum(counts), len(counts), K, rank, N)
            down.add(("apart" if plan.apart else 1 if rank <= 16 else 2 if rank <= 32 else 4 if rank <= 64 else 8, K % 2 == 0))
            kernel = min(int(rules[p].steps(rank)), 3) if plan.diagonals else "tile"
            mode = "narrow" if N % 2 else "past the caches" if plan.streams else "pairs"
            up.add((kernel, mode))
            if shape in STREAMED:
                assert mode == "past the caches", shape
                streamed.add((kernel, plan.grouped))
        assert down == {(w, even) for w in ("apart", 1, 2, 4, 8) for even in (False, True)}
        assert up == {(k, m) for k in (1, 2, 3, "tile") for m in ("narrow", "pairs", "past the caches")}
        assert {(2, True), ("tile", True)} <= streamed


def test_every_variant_of_sampling_has_its_rows(rules):
    for lib in rules.values():
        opened, alone = set(), set()
        for rows, vocab, m in SAMPLED + [SAMPLED_STREAMED]:
            if lib.sample(rows, vocab, (1 << 64) - 1).small:
                alone.add(vocab <= 8192)
            else:
                opened.add((vocab % 2 == 0, m * rows * vocab * 8 > lib.streamed()))
        assert alone == {False, True} and opened == {(even, past) for even in (False, True) for past in (False, True)}


@gpu
@pytest.mark.parametrize("shape", ODD, ids=lambda s: f"{s[0]}-{s[1]}-{s[2]}")
@pytest.mark.parametrize("n,t,p,f", [(3, 1, P61, 13), (5, 2, P61, 13), (7, 3, P61, 13), (3, 1, P45, 12), (6, 2, P45, 12)])
def test_odd_lengths_and_widths(n, t, p, f, shape):
    K, N, rank, counts, index = shape
    rng = np.random.default_rng(K + n)
    sets, tokens = make(n, t, p, f, K, N, rank, 3, rng), sum(counts)
    x, base = uniform((n, tokens, K), p, rng), uniform((n, tokens, N), p, rng)
    ss = SSNet(n, t, f=f, seed=11, p=p)
    start = i32(np.concatenate([[0], np.cumsum(counts)]).tolist())
    got = ss.adapters_mod(load(ss, sets, K, rank, N), dev(x), start, i32(index), 5, base=dev(base))
    assert np.array_equal(host(got), reference(x, sets, counts, index, base, n, t, f, p, 11, 5))


@gpu
@pytest.mark.parametrize("shape", STREAMED, ids=lambda s: f"{len(s[3])}-{s[2]}")
@pytest.mark.parametrize("p", SCHEMES, ids={P61: "p61", P45: "p45"}.get)
def test_second_products_past_the_caches(p, shape):
    """some rows against the oracle; all of them against the call whose tensors have gaps of one element, which goes through the caches, against the
    one in place, and against the one without a base"""
    K, N, rank, counts, index = shape
    n, t, f = SCHEMES[p]
    rng = np.random.default_rng(rank + len(counts))
    sets, tokens = make(n, t, p, f, K, N, rank, 3, rng), sum(counts)
    x = uniform((n, tokens, K), p, rng)
    gen = torch.Generator(device="cuda").manual_seed(rank)
    base = torch.randint(0, p, (n, tokens, N), generator=gen, device="cuda")
    base[:, ::7, 100:108] = dev(EDGES(p))
    ss = SSNet(n, t, f=f, seed=11, p=p)
    held, args = load(ss, sets, K, rank, N), (i32(np.concatenate([[0], np.cumsum(counts)]).tolist()), i32(index), 5)
    got = ss.adapters_mod(held, dev(x), *args, base=base)

    # of the first and the last tile, of its neighbours, and around the requests' ends
    ends = np.cumsum(counts)[[0, len(counts) // 2, -2]]
    picks = sorted({r for e in (0, 16, 64, 512, tokens, *ends.tolist()) for r in range(e - 2, e + 2) if 0 <= r < tokens})
    place = np.repeat(index, counts)
    z2 = np.zeros((n, tokens, rank), np.uint64)
    for i, (a, _) in enumerate(sets):
        z2[:, place == i] = orc.linear(np.ascontiguousarray(x[:, place == i]), a, p)
    z = orc.truncate(orc.degree_reduce(z2.reshape(n, -1), n, t, p, 11, 5), n, t, f, p, 11, 5).reshape(n, tokens, rank)
    want = host(base[:, picks].contiguous()).copy()
    for j, r in enumerate(picks):
        if place[r] >= 0:
            want[:, j] = (want[:, j] + orc.linear(np.ascontiguousarray(z[:, r:r + 1]), sets[place[r]][1], p)[:, 0]) % np.uint64(p)
    assert {int(place[r]) for r in picks} >= {-1, 0, 2}
    assert np.array_equal(host(got[:, picks].contiguous()), want)

    gaps, out = (torch.full((n, tokens, N + 1), -7, dtype=torch.int64, device="cuda") for _ in range(2))
    gaps[:, :, :N] = base
    ss.adapters_mod(held, dev(x), *args, base=gaps[:, :, :N], out=out[:, :, :N])
    assert torch.equal(got, out[:, :, :N]) and bool((out[:, :, N] == -7).all())
    alone = ss.adapters_mod(held, dev(x), *args)
    assert torch.equal((alone + base) % p, got)
    assert ss.adapters_mod(held, dev(x), *args, base=base, out=base) is base and torch.equal(base, got)


@gpu
@pytest.mark.parametrize("p", SCHEMES, ids={P61: "p61", P45: "p45"}.get)
def test_logits_past_the_caches_in_pairs(p):
    n, t, f = SCHEMES[p]
    rows, vocab, m = SAMPLED_STREAMED
    rng = np.random.default_rng(rows)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    picked = [0, 1, rows // 2, rows - 1]
    values = np.rint(rng.standard_normal((len(picked), vocab)) * 3 * 2 ** f).astype(np.int64)
    values[1] >>= f                             # few different ones
    shares = dev(orc.share((values % p).astype(np.uint64), n, t, p, 5, 6))
    logits = torch.zeros((n, rows, vocab), dtype=torch.int64, device="cuda")
    for i, r in enumerate(picked):
        logits[:, r] = shares[:, i]
    random = torch.from_numpy(rng.integers(0, 1 << 62, rows)).cuda()
    for params in ((0.8, 50, 0.9, 0.0), (1.3, 0, 0.97, 0.01)):
        how = fx.sampling_parameters(*params, rows=rows, device="cuda")
        tokens, shown = ss.sample(logits, list(range(1, m + 1)), how, random)
        for i, r in enumerate(picked):
            assert (int(tokens[r]), int(shown[r])) == draw(kept_weights(values[i], f, how[0].tolist()), int(random[r])), (params, r)


def test_the_room_of_more_rows_serves_fewer(rules):
    """Where rows go in several runs as well: a smaller call is never refused, stays in its room, and goes in one run where its rows fit what a run may take."""
    run = 512 << 20
    several = 0
    for lib in rules.values():
        for vocab in (100, 8193, 16384, 32000, 32768, 32769, 128000, 1 << 20):
            for most in (2, 128, 256, 300, 1000, 5000):
                room = lib.sample(most, vocab, (1 << 64) - 1).bytes
                for rows in {1, 2, most // 7, most // 2, min(200, most), min(256, most), most - 1, most} - {0}:
                    p = lib.sample(rows, vocab, room)
                    assert p.slab >= 1 and (p.small or p.bytes <= room)
                    if p.small:
                        assert p.slab == rows
                        continue
                    row = p.bytes // p.slab
                    assert row * p.slab == p.bytes and p.slab == min(rows, run // row, ((1 << 24) - 1) // p.opens // 4)
                    several += p.slab < rows
    assert several


def test_tokens_of_no_request_have_tiles(rules):
    """of the first product, whose planes the reduction sends: tiles of 16 of each request's tokens and of the others together"""
    rng = np.random.default_rng(5)
    spare = set()
    for lib in rules.values():
        for _ in range(2000):
            requests = int(2 ** rng.uniform(0, 7))
            counts = rng.integers(0, rng.integers(2, 80), requests)
            others = int(rng.integers(0, 50))
            tokens = int(counts.sum()) + others
            if not tokens:
                continue
            plan = lib.adapters(3, 1, tokens, requests, 256, 16, 64)
            need = tokens if plan.grouped else int((-(-counts // 16)).sum()) + -(-others // 16)
            assert need <= plan.down_tiles <= tokens
            spare.add(plan.down_tiles - need)
    assert 0 in spare
