"""What the messages of attention tell the party that opens them: sums of a row's scores and one mask, and nothing else of the products they
come from."""
import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61
from test_attention import Context, fixed_scale, host, shares_of

gpu = pytest.mark.gpu


def rank(matrix, p):
    """of a matrix of field elements"""
    rows, found = [[int(v) % p for v in row] for row in matrix], 0
    for col in range(len(rows[0])):
        pivot = next((r for r in range(found, len(rows)) if rows[r][col]), None)
        if pivot is None:
            continue
        rows[found], rows[pivot] = rows[pivot], rows[found]
        inverse = pow(rows[found][col], -1, p)
        for r in range(found + 1, len(rows)):
            if rows[r][col]:
                factor = rows[r][col] * inverse % p
                rows[r] = [(a - factor * b) % p for a, b in zip(rows[r], rows[found])]
        found += 1
    return found


def differences(messages, p):
    """messages [rows][keys] of one party -> what is left of them once a mask that is the same for a row is taken off"""
    m = messages.astype(object)
    return (m[:, 1:] - m[:, :1]) % p


def check_messages(msg, n, t, p, dim):
    """msg [2t+1][rows][keys], more rows and keys than dim: a party's scores q . k have the rank dim at most, whatever is added to their rows, and with
    it queries and keys could be taken from them; uniform ones have the full rank (but for a chance of 2^-44)"""
    rows, keys = msg.shape[1:]
    assert rows > dim and keys > rows + 1
    lam = orc.lagrange(list(range(1, 2 * t + 2)), p).astype(object)
    for i in range(2 * t + 1):
        assert rank(differences(msg[i], p), p) == rows
    # nor do any 2t of the parties together give more away, in the combination that would open a product of a smaller degree
    for left_out in (0, 2 * t):
        ids = [i + 1 for i in range(2 * t + 1) if i != left_out]
        part = sum(int(c) * msg[i - 1].astype(object) for c, i in zip(orc.lagrange(ids, p), ids)) % p
        assert rank(differences(part, p), p) == rows
    # what they are for: all together open to the scores and the row's mask
    opened = sum(int(c) * msg[i].astype(object) for i, c in enumerate(lam)) % p
    assert rank(differences(opened, p), p) == dim


@pytest.mark.parametrize("n,t,p,f", [(3, 1, P61, 13), (5, 2, P61, 13), (3, 1, P45, 12), (8, 3, P45, 12)])
def test_messages_of_the_oracle_hide_queries_and_keys(n, t, p, f):
    rng = np.random.default_rng(2)
    c, heads, dim, length = 10, 2, 16, 24
    q, k, v = (shares_of(rng.standard_normal(s), n, t, f, p, i) for i, s in ((1, (c, heads, dim)), (2, (length, 1, dim)), (3, (length, 1, dim))))
    _, msg, _, _ = orc.attention(q, k, v, t, f, fixed_scale(dim), f, False, p, 9, 4, full=True)
    check_messages(msg.reshape(2 * t + 1, c * heads, length), n, t, p, dim)


@gpu
@pytest.mark.parametrize("n,t,p,f", [(3, 1, P61, 13), (5, 2, P61, 13), (3, 1, P45, 12), (8, 3, P45, 12)])
@pytest.mark.parametrize("length", [24, 300])
def test_messages_hide_queries_and_keys(n, t, p, f, length):
    c = Context(n, t, p, f, [10], [length], 2, 1, 16, 16)
    c.run(f, causal=False)
    keys = (length + 63) // 64 * 64
    msg = host(c.ss.messages())[:(2 * t + 1) * 20 * keys].reshape(2 * t + 1, 20, keys)
    assert np.array_equal(msg[:, :, :length], c.want(f, False, full=True)[0][1].reshape(2 * t + 1, 20, length))
    check_messages(msg[:, :, :24], n, t, p, 16)


@gpu
@pytest.mark.parametrize("n,t,p,f,chunk,length,heads", [(5, 2, P61, 13, 600, 2000, 8), (3, 1, P45, 12, 1, 4500, 3), (7, 3, P61, 13, 40, 200, 6)])
def test_messages_of_every_kernel_are_the_oracles(n, t, p, f, chunk, length, heads):
    """tiles of 16 and of 32 rows, the share of the last party among them, keys from every part of a row"""
    c = Context(n, t, p, f, [chunk], [length], heads, 1, 32, 16)
    c.run(f)
    keys = (length + 63) // 64 * 64
    last = min(chunk, 2)
    msg = host(c.ss.messages()[:(2 * t + 1) * chunk * heads * keys].view(2 * t + 1, chunk, heads, keys)[:, -last:])
    c.q[0] = c.q[0][:, -last:]
    _, want, _, _ = orc.attention(c.q[0], c.k[0], c.v[0], t, f, fixed_scale(32), f, True, p, 21, 5, chunk - last, full=True)
    for i in range(last):
        seen = length - last + i + 1
        assert np.array_equal(msg[:, i, :, :seen], want[:, i, :, :seen])


@gpu
@pytest.mark.parametrize("n,t,p,f,chunks,lengths,heads", [(3, 1, P61, 13, [5], [40], 2), (5, 2, P61, 13, [30, 1, 0, 50], [90, 17, 5, 30], 3),
                                                          (3, 1, P45, 12, [3], [4500], 1), (5, 2, P61, 13, [600], [2000], 8)])
@pytest.mark.parametrize("causal", [True, False])
def test_scores_of_keys_that_a_row_does_not_see_are_not_sent(n, t, p, f, chunks, lengths, heads, causal):
    """under the row's mask, the opening party would learn them: of later tokens, and of what unused places held"""
    c = Context(n, t, p, f, chunks, lengths, heads, 1, 16, 16)
    ss, tokens = c.ss, sum(chunks)
    ss.reserve(ss.workspace_bytes_attention(c.cache, len(chunks), tokens, heads, max(lengths)))
    ss.messages().fill_(-1)                            # no field element
    c.run(f, causal)
    keys = (max(lengths) + 63) // 64 * 64
    sent = (ss.messages()[:(2 * t + 1) * tokens * heads * keys].view(2 * t + 1, tokens, heads, keys) != -1).cpu().numpy()
    at = 0
    for count, length in zip(chunks, lengths):
        for i in range(count):
            seen = max(0, length - count + i + 1) if causal else length
            assert sent[:, at, :, :seen].all() and not sent[:, at, :, seen:].any(), (at, seen)
            at += 1
