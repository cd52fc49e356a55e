"""Calls of the 8-bit cache's operators that their documentation allows: none of them goes through the shapes of
``test_gpu_kv8.py``.  Tolerances are that file's."""
import sys

import numpy as np
import pytest

from oracle import kv8_oracle as ko
from tests.test_gpu_kv8 import Setup, _check_attend, _check_values, _eps, _i32, _np, corun, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


def _decode_call(torch, s, n_q, seed=0, dtype="bfloat16"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(s.table.shape[0], n_q, s.hd, generator=g) * 0.1).to(getattr(torch, dtype)).cuda()


# ---------------------------------------------------------------- calls without tokens

def test_calls_without_tokens(torch, corun):
    """A step in which no row brings a token: nothing is read or written, nothing raised."""
    s = Setup(torch, corun, [40, 7], 2, 64, 16, seed=1)
    before = s.state()
    ctx, cu = _i32(torch, [40, 7]), _i32(torch, [0, 0, 0])
    empty = lambda heads: torch.empty(0, heads, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    mass = torch.full((2, 2, s.max_blocks * 16), 3.0, device="cuda")
    assert s.cache.append(empty(2), empty(2), ctx, s.t_table, cu=cu, mass=mass) is None
    q = s.cache.append(empty(2), empty(2), ctx, s.t_table, cu=cu, positions=pos, rope=corun.Rope(64), q=empty(8), mass=mass)
    assert q.shape == (0, 8, 64)
    att = corun.Kv8Attention(2, 8, 2, 64, s.max_blocks, 16, tokens=8, max_new=4)
    assert att.run(q, s.cache, ctx, s.t_table, 0.1, cu=cu, mass=mass).shape == (0, 8, 64)
    att.sync()
    # behind a call with tokens, too
    x = _decode_call(torch, s, 8)
    att.run(x, s.cache, ctx, s.t_table, 0.1, cu=_i32(torch, [0, 1, 2]))
    att.run(q, s.cache, ctx, s.t_table, 0.1, cu=cu, mass=mass)
    att.sync()
    after = s.state()
    assert np.array_equal(before[0], after[0]) and np.array_equal(before[1], after[1]) and bool((mass == 3).all())


# ---------------------------------------------------------------- calls of the binding

def test_one_token_each_where_more_are_allowed(torch, corun):
    """An object made for several tokens a row serves a call without cu (one token each), with the same bytes."""
    s = Setup(torch, corun, [300, 0, 17], 2, 128, 16, seed=2)
    q, ctx = _decode_call(torch, s, 8), _i32(torch, [300, 0, 17])
    want = corun.Kv8Attention(3, 8, 2, 128, s.max_blocks).run(q, s.cache, ctx, s.t_table, 0.1)
    for max_new in (4, 100):
        att = corun.Kv8Attention(3, 8, 2, 128, s.max_blocks, tokens=100, max_new=max_new)
        assert torch.equal(att.run(q, s.cache, ctx, s.t_table, 0.1), want)
        att.sync()
        # with weights: a row's own columns count, not those of the largest call
        mass = torch.zeros(3, 2, s.max_blocks * 16, device="cuda")
        assert torch.equal(att.run(q, s.cache, ctx, s.t_table, 0.1, mass=mass), want)
        att.sync()
        got = _np(mass.sum(-1))                                 # 4 heads of a key head; each weight within 2^-21 or so of its own
        assert np.all(np.abs(got - np.array([[4.0], [0.0], [4.0]])) <= 4 * (2.0 ** -16 + 300 * 2.0 ** -24))


def test_sync_waits_for_the_call(torch, corun):
    """``sync`` waits for the last call whatever stream is current, and behind a replay for the current stream."""
    s = Setup(torch, corun, [300, 17], 2, 64, 16, seed=3)
    q, ctx = _decode_call(torch, s, 8), _i32(torch, [300, 17])
    att = corun.Kv8Attention(2, 8, 2, 64, s.max_blocks)
    want = att.run(q, s.cache, ctx, s.t_table, 0.1)
    att.sync()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                          # some 100 ms
        out = att.run(q, s.cache, ctx, s.t_table, 0.1)
    att.sync()
    assert side.query() and torch.equal(out, want)
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.graph(g):
        torch.cuda._sleep(200_000_000)
        att.run(q, s.cache, ctx, s.t_table, 0.1, out=out)
    g.replay()
    att.sync()
    assert torch.cuda.current_stream().query() and torch.equal(out, want)


def test_append_without_out_leaves_zeros(torch, corun):
    """The queries that ``append`` returns: zeros for tokens of no row, whatever the memory held before."""
    s = Setup(torch, corun, [40, 0, 7], 2, 128, 16, seed=4)
    x = _decode_call(torch, s, 12)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    used = torch.full((3, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    del used                                                    # its memory is the next call's
    out = s.cache.append(k, v, _i32(torch, [40, 0, 7]), s.t_table, q=q)
    assert torch.equal(out[::2], q[::2]) and bool((out[1] == 0).all())


@pytest.mark.parametrize("window", [2 ** 30, 2 ** 31, 2 ** 32, 2 ** 32 + 5, sys.maxsize])
def test_windows_beyond_the_cache(torch, corun, window):
    """A window wider than any cache is no window."""
    s = Setup(torch, corun, [300, 17], 2, 64, 16, seed=5)
    q, ctx = _decode_call(torch, s, 8), _i32(torch, [300, 17])
    att = corun.Kv8Attention(2, 8, 2, 64, s.max_blocks)
    want = att.run(q, s.cache, ctx, s.t_table, 0.1)
    assert torch.equal(att.run(q, s.cache, ctx, s.t_table, 0.1, window=window), want)
    with pytest.raises(corun.CorunError):
        att.run(q, s.cache, ctx, s.t_table, 0.1, window=-window)


def test_workspace_is_held_once(torch, corun):
    """Between two calls of an object there is one workspace, while the second runs there is no more than one."""
    s = Setup(torch, corun, [3000] * 4, 4, 128, 16, seed=6)
    q, ctx = _decode_call(torch, s, 32), _i32(torch, [3000] * 4)
    out = torch.zeros_like(q)
    att = corun.Kv8Attention(4, 32, 4, 128, s.max_blocks)
    att.run(q, s.cache, ctx, s.t_table, 0.1, out=out)
    att.sync()
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    att.run(q, s.cache, ctx, s.t_table, 0.1, out=out)
    att.sync()
    from paper_2608_14376_b200.corun import lib
    size = lib().corun_kv8_attend_bytes(4, 4, 1, 32, 4, 128, 16, s.max_blocks, 0)
    assert torch.cuda.memory_allocated() <= held and torch.cuda.max_memory_allocated() < held + size // 2


# ---------------------------------------------------------------- numbers

def _one_token_takes_all(torch, corun, G, hd, n, scale, sign):
    """Only the first dim of queries and keys is not 0, so a score is one product; the largest one is apart from the others by at least
    1.25 * scale, and its token takes all the weight."""
    c, n_kv = 300, 2
    s = Setup(torch, corun, [c], n_kv, hd, 16, seed=7)
    codes, exps = s.codes.copy(), s.exps.copy()
    codes[:, 0], exps[:, 0] = 0, 0
    far = int(s.rng.integers(0, c - n + 1))                     # (seen by every query of the call)
    for j in range(c):                                          # 1 or 256 for one token, 2.25 to 240 for the others
        codes[s.table[0, j // 16], 0, :, j % 16, 0] = (0x38 if sign < 0 else 0x78) if j == far else 0x41 + int(s.rng.integers(0, 0x37))
    s.cache.pool.copy_(torch.tensor(codes).cuda().view(torch.float8_e4m3fn))
    s.cache.exps.copy_(torch.tensor(exps))
    s.want = ko.Cache(codes, exps)
    q = torch.zeros(n, G * n_kv, hd, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = sign
    att = corun.Kv8Attention(1, G * n_kv, n_kv, hd, s.max_blocks, tokens=n, max_new=n)
    out = att.run(q, s.cache, _i32(torch, [c]), s.t_table, scale, cu=_i32(torch, [0, n]))
    att.sync()
    v = np.repeat(s.want.values(s.table[0], c)[1][far], G, 0)
    # one weight of 1: what is left is its rounding with the value's (11 bits, the sum of weights alike) and the output's
    assert np.all(np.abs(_np(out) - v) <= (_eps(torch, torch.bfloat16) + 2 * 2.0 ** -11) * np.abs(v))


HUGE = [1e6, 1e8, 3e8, 1e9, 1e20, 1e32]


@pytest.mark.parametrize("G,hd,n", [(4, 128, 1), (8, 64, 1), (16, 128, 1), (2, 128, 3)])
@pytest.mark.parametrize("scale", HUGE)
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_attend_huge_scores(torch, corun, G, hd, n, scale, sign):
    _one_token_takes_all(torch, corun, G, hd, n, scale, sign)


@pytest.mark.parametrize("G,hd,n", [(8, 128, 9), (4, 64, 20)])
@pytest.mark.parametrize("scale", HUGE)
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_chunk_huge_scores(torch, corun, G, hd, n, scale, sign):
    _one_token_takes_all(torch, corun, G, hd, n, scale, sign)
