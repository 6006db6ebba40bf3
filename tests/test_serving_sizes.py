"""How calls with adapters and of sampling are cut up (csrc/serving_plan.hpp, compiled for the host, so that a rule that changes does not leave a kernel
without its test), and memories of more than 4 GB."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import Adapters, P45, P61, SSNet
from paper_2406_02629_amd import fixedpoint as fx
from test_adapters import SHAPES, dev, host, i32, make, reference, uniform
from test_sampling import draw, kept_weights

gpu = pytest.mark.gpu
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_02629_amd", "csrc")
sz = C.c_size_t


class AdapterPlan(C.Structure):
    _fields_ = [("grouped", C.c_bool), ("apart", C.c_bool), ("diagonals", C.c_bool), ("splits", C.c_int), ("run", C.c_int), ("streams", C.c_bool), ("col_groups", C.c_int)] + \
               [(k, sz) for k in ("messages", "planes", "z", "down_tiles", "up_tiles", "down_groups", "up_groups", "bytes")]


class SamplePlan(C.Structure):
    _fields_ = [("small", C.c_bool)] + [(k, C.c_int) for k in ("slab", "opens", "groups", "chunks", "key_ld")] + [("bytes", sz)]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d, libs = tmp_path_factory.mktemp("serving_plan"), {}
    src = d / "serving_plan.cpp"
    src.write_text('#include "serving_plan.hpp"\nextern "C" {\n'
                   "SS_NS::adapter_plan adapters(int n, int t, int tokens, int requests, int K, int rank, int N)\n"
                   "{ return SS_NS::plan_adapters(n, t, tokens, requests, K, rank, N); }\n"
                   "SS_NS::sample_plan sample(int rows, int vocab, size_t room) { return SS_NS::plan_sample(rows, vocab, room); }\n"
                   "size_t tiles(size_t tokens, size_t requests, size_t rows) { return SS_NS::request_tiles(tokens, requests, rows, false); }\n}\n")
    for p, limbs in ((P61, 8), (P45, 6)):
        so = str(d / f"serving_plan{limbs}.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-DSS_NLIMB={limbs}", "-DSS_NS=rules", "-I", CSRC, "-o", so,
                        str(src)], check=True)
        lib = libs[p] = C.CDLL(so)
        lib.adapters.restype, lib.adapters.argtypes = AdapterPlan, [C.c_int] * 7
        lib.sample.restype, lib.sample.argtypes = SamplePlan, [C.c_int, C.c_int, sz]
        lib.tiles.restype, lib.tiles.argtypes = sz, [sz] * 3
    return libs


def test_shapes_of_the_tests_take_every_kernel(rules):
    seen = set()
    for p, (n, t) in ((P61, (5, 2)), (P45, (3, 1))):
        for K, N, rank, counts, _ in SHAPES:
            plan = rules[p].adapters(n, t, sum(counts), len(counts), K, rank, N)
            width = 1 if rank <= 16 else 2 if rank <= 32 else 4 if rank <= 64 else 8      # columns of A among the waves, see ss_launch_adapters_down
            seen |= {(p, "down", width), (p, "apart", plan.apart, K % 2 == 0), (p, "grouped", plan.grouped, plan.diagonals), (p, "runs", plan.splits > 1), (p, "steps", -(-rank // 8) if rank <= 8 else -(-rank // 16), plan.diagonals),
                     (p, "parts", plan.col_groups > 1)}
    for p in (P61, P45):
        assert {(p, "down", w) for w in (1, 2, 4, 8)} | {(p, "apart", a, w) for a in (False, True) for w in (False, True)} | {(p, "grouped", a, b) for a in (False, True) for b in (False, True)} <= seen
        assert {(p, "runs", False), (p, "runs", True), (p, "parts", False), (p, "parts", True), (p, "steps", 1, True), (p, "steps", 2, True)} <= seen


def test_a_plan_covers_its_call(rules):
    rng = np.random.default_rng(1)
    for lib in rules.values():
        for _ in range(3000):
            n, t = [(3, 1), (5, 2), (8, 3)][rng.integers(3)]
            requests, K, rank, N = int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 13.99)), int(rng.integers(1, 129)), int(2 ** rng.uniform(0, 20))
            tokens = max(1, int(requests * 2 ** rng.uniform(-1, 6)))
            p = lib.adapters(n, t, tokens, requests, K, rank, N)
            blocks = -(-K // 64)
            assert 1 <= p.splits <= 8 and (p.splits - 1) * p.run < blocks <= p.splits * p.run and p.run * 64 <= 16384
            assert p.col_groups >= 1 and n * p.col_groups < 65536 and p.grouped <= (requests <= 1024)
            assert p.bytes == p.messages + p.planes + p.z and p.planes >= p.splits * (2 * t + 1) * tokens * rank * 8 and p.z >= n * tokens * rank * 8
            assert p.down_groups == (-(-p.down_tiles // 4) if p.apart else p.down_tiles) * (2 * t + 1) * p.splits and p.apart <= (rank <= 16) and p.up_groups == p.up_tiles * n * p.col_groups
        for _ in range(300):
            counts = rng.integers(0, 70, rng.integers(1, 30))
            if counts.sum():
                for rows in (16, 64):
                    assert int((-(-counts // rows)).sum()) <= lib.tiles(int(counts.sum()), counts.size, rows)


def test_rows_that_are_sampled_together_fit_the_room(rules):
    lib = rules[P61]
    for rows in (1, 7, 256, 5000, 1 << 20):
        for vocab in (1, 8192, 8193, 32000, 200003, 1 << 20):
            p = lib.sample(rows, vocab, (1 << 64) - 1)
            assert 1 <= p.slab <= rows and p.small >= (vocab <= 8192) and p.small <= (vocab <= 32768)
            if p.small:
                assert p.slab == rows and (p.bytes == 0) == (vocab <= 8192) and lib.sample(rows, vocab, 0).slab == rows
                continue
            assert p.opens * 1024 >= vocab > (p.opens - 1) * 1024 and p.chunks * 512 >= vocab > (p.chunks - 1) * 512 and p.chunks <= 2048
            assert vocab <= p.key_ld < vocab + 4 and p.key_ld % 4 == 0 and 16 * p.groups <= p.chunks + 15
            assert p.slab * p.opens < 1 << 24 and p.bytes <= max(512 << 20, p.bytes // p.slab)
            one = p.bytes // p.slab
            assert lib.sample(rows, vocab, one - 1).slab == 0 and lib.sample(rows, vocab, one).slab == 1


def test_the_room_of_a_larger_call_holds_smaller_ones(rules):
    rng = np.random.default_rng(3)
    for lib in rules.values():
        for _ in range(300):
            n, t = [(3, 1), (5, 2), (8, 3)][rng.integers(3)]
            K, rank, N, most = int(2 ** rng.uniform(0, 13.99)), int(rng.integers(1, 129)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 12))
            room = lib.adapters(n, t, most, 16, K, rank, N).bytes
            for tokens in rng.integers(1, most + 1, 8).tolist() + [1, most]:
                for requests in (1, 5, 16, 2000):
                    assert lib.adapters(n, t, tokens, requests, K, rank, N).bytes <= room
        for vocab in (100, 8193, 16384, 32000, 32768, 32769, 128000, 1 << 20):
            for most in (2, 128, 256, 300, 1000):
                room = lib.sample(most, vocab, (1 << 64) - 1).bytes
                for rows in {1, most - 1, most // 2, min(256, most), min(200, most), most}:
                    p = lib.sample(rows, vocab, room)
                    assert p.bytes <= room and p.slab == rows or most * vocab > 1 << 26


@gpu
def test_a_set_of_more_than_4_gb():
    n, t, p, f, K, N, rank, places = 3, 1, P61, 13, 4096, 3000, 16, 3000
    rng = np.random.default_rng(2)
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = Adapters(ss, places, K, rank, N)
    assert held.down.numel() > 1 << 32 and held.up.numel() > 1 << 31
    sets = make(n, t, p, f, K, N, rank, 2, rng)
    held.load(places - 1, dev(sets[1][0]), dev(sets[1][1])), held.load(0, dev(sets[0][0]), dev(sets[0][1]))
    counts, index = [3, 20, 1], [places - 1, 0, places - 1]
    x, base = uniform((n, 24, K), p, rng), uniform((n, 24, N), p, rng)
    want = reference(x, sets, counts, [1, 0, 1], base, n, t, f, p, 3, 5)
    assert np.array_equal(host(ss.adapters_mod(held, dev(x), i32([0, 3, 23, 24]), i32(index), 5, base=dev(base))), want)


@gpu
def test_logits_of_more_than_4_gb_in_several_runs():
    """rows beyond 2^32 bytes of a share and keys in more than one run of rows: the first and last row of each run and of the call"""
    f, vocab, rows = 13, 100001, 2000
    rng = np.random.default_rng(3)
    ss = SSNet(3, 1, f=f, seed=3)
    logits = torch.zeros((3, rows, vocab), dtype=torch.int64, device="cuda")
    params = fx.sampling_parameters(0.8, 50, 0.875, rows=rows, device="cuda")
    random = torch.from_numpy(rng.integers(0, 1 << 62, rows)).cuda()
    picked = [0, 1, 600, 1100, 1200, rows - 2, rows - 1]
    values = np.rint(rng.standard_normal((len(picked), vocab)) * 3 * 2 ** f).astype(np.int64)
    shares = dev(orc.share((values % P61).astype(np.uint64), 3, 1, P61, 5, 6))
    for i, r in enumerate(picked):
        logits[:, r] = shares[:, i]
    tokens, shown = ss.sample(logits, [1, 3], params, random)
    for i, r in enumerate(picked):
        assert (int(tokens[r]), int(shown[r])) == draw(kept_weights(values[i], f, params[0].tolist()), int(random[r]))
    # rows of equal logits: of the first 50 as many stay as 0.875 of them need, 43.75, so 44, in equal parts
    equal = [r for r in range(rows) if r not in picked]
    want = np.array([int(random[r]) * 44 >> 62 for r in equal])
    assert np.array_equal(tokens[equal].cpu().numpy(), want)


@gpu
@pytest.mark.parametrize("p,rows,vocab,small", [(P61, 256, 32768, True), (P61, 250, 9000, True), (P45, 200, 16001, True), (P61, 256, 32769, False), (P61, 3, 8193, False)])
def test_rows_in_one_launch_and_in_four(rules, p, rows, vocab, small):
    """either side of the rules, every kind of cut among the rows that are looked at"""
    assert rules[p].sample(rows, vocab, (1 << 64) - 1).small == small
    f = 13 if p == P61 else 12
    rng = np.random.default_rng(vocab)
    ss = SSNet(3, 1, f=f, seed=3, p=p)
    picked = sorted({0, 1, rows // 2, rows - 2, rows - 1})      # each once: of three rows 0, 1, 2
    values = np.rint(rng.standard_normal((len(picked), vocab)) * 3 * 2 ** f).astype(np.int64)
    values[-1] >>= 13                           # few different ones
    shares = dev(orc.share((values % p).astype(np.uint64), 3, 1, p, 5, 6))
    logits = torch.zeros((3, rows, vocab), dtype=torch.int64, device="cuda")
    for i, r in enumerate(picked):
        logits[:, r] = shares[:, i]
    random = torch.from_numpy(rng.integers(0, 1 << 62, rows)).cuda()
    for params in ((0.8, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.3, 0, 0.97, 0.01), (0.5, 700, 1.0, 0.0)):
        how = fx.sampling_parameters(*params, rows=rows, device="cuda")
        tokens, shown = ss.sample(logits, [1, 2], how, random)
        for i, r in enumerate(picked):
            assert (int(tokens[r]), int(shown[r])) == draw(kept_weights(values[i], f, how[0].tolist()), int(random[r])), (params, r)
