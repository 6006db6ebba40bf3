"""What adapters send: nothing of what the workspace held before."""
import numpy as np
import pytest
import torch

import oracle as orc
from paper_2406_02629_amd import P45, P61, SSNet, binding
from test_adapters import dev, host, i32, load, make, uniform

gpu = pytest.mark.gpu

# (tokens, start, places): tokens in front of the first request or behind the last belong to none
PADDED = [
    (40, [0, 21], [0]),
    (18, [0, 17], [1]),                                            # as many tiles as the requests alone may have
    (8, [2, 3, 4, 5], [0, 1, 0]),
    (300, [5, 5, 130, 262], [1, 0, 2]),
    (20, [0, 0], [0]),                                             # of none at all
    (20, [99, 99], [0]),
    (33, list(range(25)), [i % 4 - 1 for i in range(24)]),         # single tokens that share adapters
    (150, [3] + list(range(3, 103)), [0] * 100),
    (3001, [7, 2950], [0]),                                        # a wave to a tile of the first product
    (4000, [0, 2100, 2100, 3900], [1, 0, 2]),
]


@gpu
@pytest.mark.parametrize("tokens,start,index", PADDED, ids=[f"{c[0]}-{len(c[2])}" for c in PADDED])
@pytest.mark.parametrize("n,t,p,f,K,rank", [(5, 2, P61, 13, 800, 9), (3, 1, P61, 13, 64, 40), (3, 1, P45, 12, 100, 16)])
def test_tokens_of_no_request_send_nothing(n, t, p, f, K, rank, tokens, start, index):
    """their part of the messages is that of zeros, whatever lies in the workspace"""
    N = 34
    rng = np.random.default_rng(tokens)
    sets = make(n, t, p, f, K, N, rank, 3, rng)
    x, base = uniform((n, tokens, K), p, rng), dev(uniform((n, tokens, N), p, rng))
    ss = SSNet(n, t, f=f, seed=3, p=p)
    held = load(ss, sets, K, rank, N)
    z2 = np.zeros((n, tokens, rank), np.uint64)
    inside = np.zeros(tokens, bool)
    for first, last, i in zip(start, start[1:], index):
        at = slice(min(first, tokens), min(last, tokens))
        inside[at] = True
        if i >= 0 and x[:, at].size:
            z2[:, at] = orc.linear(np.ascontiguousarray(x[:, at]), sets[i][0], p)
    _, msg1, msg2, _ = orc.degree_reduce(z2.reshape(n, -1), n, t, p, 3, 5, full=True)
    want = np.concatenate([msg1.reshape(-1), msg2.reshape(-1)])
    ss.reserve(ss.lib.ssnet_workspace_bytes_adapters(ss._ctx, held._address, len(index), tokens))
    outs = []
    for left in (0x0123456789ABCDEF, 77):
        ss._ws[binding.WS_HEADER_BYTES:].view(torch.int64).fill_(left)
        out = torch.full_like(base, -7)
        ss.adapters_mod(held, dev(x), i32(start), i32(index), 5, base=base, out=out)
        assert np.array_equal(host(ss.messages()[:want.size]), want)
        assert bool((out[:, torch.from_numpy(~inside).cuda()] == -7).all())
        outs.append(out)
    assert torch.equal(*outs)
