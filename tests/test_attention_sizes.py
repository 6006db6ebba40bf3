"""The kernels for many tokens, heads of more than 64 elements, tiles of 32 rows, runs of long contexts and large memories, against the oracle,
bit for bit.  Which kernels a size takes is asked of the rules themselves (csrc/attention_plan.hpp, compiled for the host), so that
a rule that changes does not leave a kernel without its test."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, PagedCache, SSNet
from paper_2406_02629_amd import fixedpoint as fx
from test_attention import Context, dev, fixed_scale, host, i32, shares_of

gpu = pytest.mark.gpu
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_02629_amd", "csrc")


class Plan(C.Structure):
    _fields_ = [(k, C.c_int) for k in ("row_tiles", "slab", "splits", "run", "key_block", "dblocks")] + [("finish", C.c_bool)] + \
               [(k, C.c_size_t) for k in ("keys", "rows", "bytes")] + [("split_rows", C.c_bool), ("query_bytes", C.c_size_t)]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d, libs = tmp_path_factory.mktemp("attention_plan"), {}
    src = d / "attention_plan.cpp"
    src.write_text('#include "attention_plan.hpp"\nextern "C" {\n'
                   "SS_NS::attention_plan plan(int n, int t, int tokens, int seqs, int heads, int kv, int dim, int max_length, size_t room)\n"
                   "{ return SS_NS::plan_attention(n, t, tokens, seqs, heads, kv, dim, max_length, room); }\n"
                   "bool wide_append(int tokens, int kv, int dim, int rot, size_t ld) { return SS_NS::wide_append(tokens, kv, dim, rot, ld, true); }\n"
                   "bool streams(int n, int t, int tokens, int heads, int dim, int rot)\n"
                   "{ return SS_NS::rotary_streams(n, t, tokens, heads, dim, rot) && SS_NS::wide_rotary(dim, rot, 0, heads * dim, true); }\n}\n")
    for p, limbs in ((P61, 8), (P45, 6)):
        so = str(d / f"attention_plan{limbs}.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-DSS_NLIMB={limbs}", "-DSS_NS=rules", "-I", CSRC, "-o", so,
                        str(src)], check=True)
        lib = libs[p] = C.CDLL(so)
        lib.plan.restype, lib.plan.argtypes = Plan, [C.c_int] * 8 + [C.c_size_t]
        lib.wide_append.restype, lib.wide_append.argtypes = C.c_bool, [C.c_int] * 4 + [C.c_size_t]
        lib.streams.restype, lib.streams.argtypes = C.c_bool, [C.c_int] * 6
    return libs


# ------------------------------------------------------------------ appending many tokens

SCHEMES = [(3, 1, P61, 13), (5, 2, P61, 13), (6, 2, P61, 13), (7, 3, P61, 13), (3, 1, P45, 12), (4, 1, P45, 12), (8, 3, P45, 12)]
MANY = [(620, 2, 160, 160, 32), (440, 7, 64, 24, 64), (1540, 1, 128, 0, 16), (200, 8, 128, 128, 48), (1030, 3, 64, 64, 16), (2050, 2, 48, 16, 32),
        (260, 3, 256, 96, 64)]
FEW = [(770, 2, 128, 20, 16), (1540, 1, 128, 4, 16)]      # as many elements, but their halves do not come in fours


def test_appends_take_the_kernel_they_are_for(rules):
    for lib in rules.values():
        assert all(lib.wide_append(tokens, heads, dim, rot, heads * dim) for tokens, heads, dim, rot, _ in MANY)
        assert not any(lib.wide_append(tokens, heads, dim, rot, heads * dim) for tokens, heads, dim, rot, _ in FEW)
        assert not lib.wide_append(620, 2, 160, 160, 2 * 160 + 1)


def places(order, tokens, pages, page, rng):
    if order == "scattered":
        return rng.permutation(pages * page)[:tokens]
    if order == "sequences":                   # runs of several sequences, each from its own place inside a page on
        cuts = np.sort(rng.choice(np.arange(1, tokens), 4, replace=False))
        order, slots, first = rng.permutation(pages), [], 0
        for count in np.diff(np.concatenate([[0], cuts, [tokens]])):
            at = rng.integers(0, page) + np.arange(count)
            used = at[-1] // page + 1
            slots.append(order[first + at // page] * page + at % page)
            first += used
        return np.concatenate(slots)
    start = page // 2 + 5 if order == "run" else 0
    return np.arange(tokens) + start


def put(cache, slots, k, v, digits):
    """keys and values [n, tokens, heads, dim] into the places of the cache that lie in it, as the layout says, on the GPU"""
    inside = (slots >= 0) & (slots < cache.pages * cache.page_size)
    at = torch.from_numpy(slots[inside]).cuda()
    page, cell, key = at // cache.page_size, at % cache.page_size // 16, at % 16

    def digits_of(shares):                     # tokens, n, heads, digit, dim
        return torch.from_numpy(orc.digits(shares[:, inside], digits)).cuda().permute(1, 0, 2, 4, 3)

    cache.keys[page, :, :, cell, :, :, key] = digits_of(k).unflatten(-1, (-1, 16))
    cache.values[page, :, :, cell, :, :, key] = digits_of(v)


def check_append(n, t, p, f, tokens, heads, dim, rot, page, order, layout, pages=None, far=0, part=False):
    rng = np.random.default_rng(dim + tokens)
    digits = 6 if p == P45 else 8
    k, v = (shares_of(rng.standard_normal((tokens, heads, dim)), n, t, f, p, s) for s in (3, 4))
    pages = -(-tokens // page) + 12 if pages is None else pages
    slots = places(order, tokens, pages - far, page, rng) + far * page
    slots[1], slots[-3] = -1, pages * page     # left out
    ss = SSNet(n, t, f=f, seed=21, p=p)
    cache = PagedCache(ss, pages, page, heads, dim)
    cache.keys.random_(-128, 128), cache.values.random_(-128, 128)
    want = PagedCache(ss, pages, page, heads, dim, keys=cache.keys.clone(), values=cache.values.clone())
    turned, u, wsh, kw = k, None, None, {}
    if rot:
        table, pos = fx.rotary_table(100, fx.rotary_frequencies(rot), f).numpy(), rng.integers(0, 100, tokens)
        turned, u, wsh = orc.rotary_truncate(k, table, pos, t, f, p, 21, 5, layout == "interleaved", full=True)
        kw = dict(table=torch.from_numpy(table).cuda(), pos=i32(pos.tolist()), layout=layout)
    dk, dv = dev(k), dev(v)
    if part:                                   # of the rows of a product of queries, keys and values
        rows = torch.full((n, tokens, (2 * heads + 1) * dim), -1, dtype=torch.int64, device="cuda")
        rows[:, :, dim:(heads + 1) * dim], rows[:, :, (heads + 1) * dim:] = dk.flatten(2), dv.flatten(2)
        dk, dv = (rows[:, :, a * dim:(a + heads) * dim].unflatten(-1, (heads, dim)) for a in (1, heads + 1))
    ss.cache_append(cache, dk, dv, torch.from_numpy(slots).cuda(), 5, **kw)
    put(want, slots, turned, v, digits)
    assert torch.equal(cache.keys, want.keys) and torch.equal(cache.values, want.values)
    if rot:
        msgs = host(ss.messages()[:u.size + wsh.size])
        assert np.array_equal(msgs, np.concatenate([u.reshape(-1), wsh.reshape(-1)]))


@gpu
@pytest.mark.parametrize("n,t,p,f", SCHEMES)
@pytest.mark.parametrize("tokens,heads,dim,rot,page", MANY)
@pytest.mark.parametrize("order,layout", [("cells", "half"), ("run", "interleaved"), ("scattered", "half"), ("sequences", "interleaved")])
def test_append_of_many_tokens_matches_the_oracle(n, t, p, f, tokens, heads, dim, rot, page, order, layout):
    check_append(n, t, p, f, tokens, heads, dim, rot, page, order, layout)


@gpu
@pytest.mark.parametrize("tokens,heads,dim,rot,page", MANY[:2] + FEW)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("order", ["run", "sequences"])
@pytest.mark.parametrize("p,f", [(P61, 13), (P45, 12)])
def test_append_of_many_tokens_in_either_layout_and_from_parts_of_rows(p, f, tokens, heads, dim, rot, page, layout, order):
    check_append(3, 1, p, f, tokens, heads, dim, rot, page, order, layout, part=True)


# ------------------------------------------------------------------ rotary positions past the caches

STREAMED = [(3, 1, P61, 13, 760, 33, 128, 128), (5, 2, P61, 13, 470, 33, 128, 128), (6, 2, P61, 13, 900, 11, 256, 128), (7, 3, P45, 12, 345, 33, 128, 112),
            (4, 1, P45, 12, 1001, 40, 80, 80)]


def test_rotations_take_the_kernel_they_are_for(rules):
    assert all(rules[p].streams(n, t, tokens, heads, dim, rot) for n, t, p, f, tokens, heads, dim, rot in STREAMED)
    assert not rules[P61].streams(3, 1, 700, 32, 128, 128)


@gpu
@pytest.mark.parametrize("n,t,p,f,tokens,heads,dim,rot", STREAMED)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_past_the_caches_matches_the_oracle(n, t, p, f, tokens, heads, dim, rot, layout):
    rng = np.random.default_rng(tokens)
    x = shares_of(rng.standard_normal((tokens, heads, dim)) * 4, n, t, f, p, 3)
    table, pos = fx.rotary_table(200, fx.rotary_frequencies(rot), f).numpy(), rng.integers(0, 200, tokens)
    ss = SSNet(n, t, f=f, seed=21, p=p)
    want, u, wsh = orc.rotary_truncate(x, table, pos, t, f, p, 21, 5, layout == "interleaved", full=True)
    got = ss.rotary_truncate(dev(x), torch.from_numpy(table).cuda(), i32(pos.tolist()), 5, layout=layout)
    assert torch.equal(got, dev(want))
    msgs = ss.messages()[:u.size + wsh.size]
    assert torch.equal(msgs[:u.size], dev(u.reshape(-1))) and torch.equal(msgs[u.size:], dev(wsh.reshape(-1)))
    x_in_place = dev(x)
    ss.rotary_truncate(x_in_place, torch.from_numpy(table).cuda(), i32(pos.tolist()), 5, layout=layout, out=x_in_place)
    assert torch.equal(x_in_place, got)


# ------------------------------------------------------------------ attention

# n, t, p, f, chunks, lengths, heads, heads of the cache, elements of a head, page; what of the plan the case is for
ATTENTION = [
    # values of heads of more than 64 elements, rows of one tile and of several, one run and two
    (3, 1, P61, 13, [20, 3, 41], [300, 150, 420], 12, 4, 128, 32, dict(row_tiles=1, splits=2, dblocks=2)),
    (5, 2, P61, 13, [40, 17], [400, 290], 12, 4, 128, 32, dict(row_tiles=1, splits=1, dblocks=2)),
    (5, 2, P61, 13, [40, 17], [400, 290], 12, 4, 80, 16, dict(row_tiles=1, splits=1, dblocks=2)),
    (5, 2, P45, 12, [40, 17], [400, 290], 12, 4, 112, 16, dict(row_tiles=1, splits=1, dblocks=2)),
    (7, 3, P61, 13, [33, 5], [300, 280], 4, 2, 256, 16, dict(row_tiles=1, splits=2, dblocks=4)),
    (3, 1, P45, 12, [50], [333], 4, 4, 208, 16, dict(row_tiles=1, dblocks=4)),
    # single tokens, runs of the values added up, by one wave to a result and by four
    (5, 2, P61, 13, [1, 1, 1], [900, 313, 1500], 8, 2, 128, 64, dict(row_tiles=1, dblocks=2, splits=6)),
    (3, 1, P61, 13, [1], [3300], 8, 2, 128, 64, dict(row_tiles=1, dblocks=2, splits=13)),
    (4, 1, P45, 12, [1, 1], [2900, 700], 6, 3, 192, 32, dict(row_tiles=1, dblocks=3, splits=12)),
    (3, 1, P61, 13, [1], [20000], 4, 2, 128, 64, dict(row_tiles=1, dblocks=2, split_rows=True)),
    (8, 3, P45, 12, [2], [5000], 4, 1, 96, 16, dict(row_tiles=1, dblocks=2, split_rows=True)),
    # tiles of 32 rows
    (5, 2, P61, 13, [300], [1500], 16, 2, 80, 64, dict(row_tiles=2, dblocks=2, splits=1)),
    (5, 2, P61, 13, [300], [1500], 16, 2, 128, 64, dict(row_tiles=2, dblocks=2, splits=1)),
    (3, 1, P61, 13, [400], [1999], 16, 2, 256, 64, dict(row_tiles=2, dblocks=4, splits=1, query_bytes=1 << 16)),
    (5, 2, P45, 12, [300], [1500], 16, 2, 128, 32, dict(row_tiles=2, dblocks=2, splits=1)),
    (7, 3, P45, 12, [150, 170], [900, 1100], 16, 2, 256, 32, dict(row_tiles=2, dblocks=4, splits=1)),
    (4, 1, P61, 13, [333], [2500], 15, 3, 96, 32, dict(row_tiles=2, dblocks=2, splits=1)),
    # ... rows in several workgroups, runs added up
    (5, 2, P61, 13, [33], [16500], 16, 1, 80, 64, dict(row_tiles=2, dblocks=2, splits=3, split_rows=True)),
    (3, 1, P45, 12, [60], [16400], 16, 1, 128, 64, dict(row_tiles=2, dblocks=2, splits=3, split_rows=True)),
]


def plan_of(rules, n, t, p, chunks, lengths, heads, kv, dim):
    return rules[p].plan(n, t, sum(chunks), len(chunks), heads, kv, dim, max(lengths), 8 << 30)


def test_attentions_take_the_kernels_they_are_for(rules):
    for n, t, p, f, chunks, lengths, heads, kv, dim, page, parts in ATTENTION:
        plan = plan_of(rules, n, t, p, chunks, lengths, heads, kv, dim)
        assert {k: getattr(plan, k) for k in parts} == parts and plan.slab == sum(chunks) and not plan.finish, (chunks, lengths, dim)


def check_attention(c, bits, causal=True, rows=2):
    """the last tokens of every sequence's chunk against the oracle (all of a short one)"""
    got, at = host(c.run(bits, causal)), 0
    for b, (count, length) in enumerate(zip(c.chunks, c.lengths)):
        last = min(count, rows)
        want = orc.attention(c.q[b][:, -last:], c.k[b], c.v[b], c.t, c.f, fixed_scale(c.dim), bits, causal, c.p, 21, 5, at + count - last)
        at += count
        assert np.array_equal(got[:, at - last:at], want), b


@gpu
@pytest.mark.parametrize("n,t,p,f,chunks,lengths,heads,kv,dim,page,parts", ATTENTION)
def test_attention_matches_the_oracle(n, t, p, f, chunks, lengths, heads, kv, dim, page, parts):
    c = Context(n, t, p, f, chunks, lengths, heads, kv, dim, page)
    short = max(chunks) <= 60 and max(lengths) <= 500      # all rows there
    check_attention(c, 2 * f, rows=max(chunks) if short else 2)
    if short:
        check_attention(c, f, causal=False, rows=7)


@gpu
@pytest.mark.parametrize("n,t,p,f,chunks,lengths,heads,kv,dim,page,parts", [c for c in ATTENTION if c[-1].get("row_tiles") == 2 and not c[-1].get("split_rows")])
def test_tiles_of_32_rows_give_what_tiles_of_16_give(rules, n, t, p, f, chunks, lengths, heads, kv, dim, page, parts):
    """every row: a workspace for one token takes the same tokens in small runs, whose tiles have 16 rows"""
    c = Context(n, t, p, f, chunks, lengths, heads, kv, dim, page)
    want = c.run(f)
    c.ss = SSNet(n, t, f=f, seed=21, p=p)
    c.ss.ATTENTION_ROOM = 0
    assert torch.equal(c.run(f), want)
    assert rules[p].plan(n, t, sum(chunks), len(chunks), heads, kv, dim, max(lengths), c.ss._ws.numel() - (1 << 16)).row_tiles == 1


# ------------------------------------------------------------------ memories of more than 4 GB

@gpu
@pytest.mark.parametrize("tokens,order", [(5, "scattered"), (260, "run"), (260, "scattered")])
def test_append_behind_4_gb_of_the_cache(tokens, order):
    n, heads, dim, page, pages = 3, 8, 128, 64, 2900
    assert pages * page * n * heads * dim * 8 > 1 << 32
    check_append(n, 1, P61, 13, tokens, heads, dim, 128, page, order, "half", pages=pages, far=2870)


@gpu
def test_attention_behind_4_gb_of_the_cache():
    c = Context(3, 1, P61, 13, [1, 20, 3], [700, 333, 90], 16, 8, 128, 64, extra=2900)
    assert c.cache.keys.numel() > 1 << 32 and int(c.table.max()) * c.cache.keys[0].numel() > 1 << 32
    check_attention(c, 26, rows=3)


@gpu
def test_attention_with_4_gb_of_messages(rules):
    n, t, chunk, length, heads, kv, dim = 5, 2, 512, 16384, 16, 4, 16
    assert plan_of(rules, n, t, P61, [chunk], [length], heads, kv, dim).slab < chunk
    c = Context(n, t, P61, 13, [chunk], [length], heads, kv, dim, 64)
    c.ss.ATTENTION_ROOM = 1 << 35
    check_attention(c, 26, rows=1)
    assert c.ss._ws.numel() > (2 * t + 1) * chunk * heads * length * 8 > 1 << 32
