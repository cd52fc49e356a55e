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


def _share_not_nearest(torch, corun, G, hd, n, seed):
    """The share of fp16 outputs that are not the value nearest to the exact one, and what it may be.  Three e4m3 values of a weight: each
    rounding leaves 2^-5 to 2^-4 of what it is given at most, evenly, so 2^-4.5 / sqrt(3) rms, and the third 1.7e-5 of the weight.  Values are
    positive: an output is then off by r = 1.7e-5 |p v| / sum(p v) of itself, rms.  It is rounded the other way where the middle of two
    neighbours (2^-11 of the value apart or more) lies in between: in r 2^11 of all cases, and twice that is allowed."""
    c, n_kv = 40, 4
    s = Setup(torch, corun, [c] * 3, n_kv, hd, 16, seed=seed)
    codes = s.codes.copy()
    codes[:, 1] = s.rng.integers(0x30, 0x78, codes[:, 1].shape)
    s.cache.pool.copy_(torch.tensor(codes).cuda().view(torch.float8_e4m3fn))
    s.want = ko.Cache(codes, s.exps)
    q = torch.tensor(s.rng.standard_normal((3 * n, G * n_kv, hd)) * 0.2).half().cuda()
    att = corun.Kv8Attention(3, G * n_kv, n_kv, hd, s.max_blocks, tokens=3 * n, max_new=n)
    out = att.run(q, s.cache, _i32(torch, [c] * 3), s.t_table, hd ** -0.5, cu=_i32(torch, [0, n, 2 * n, 3 * n]))
    att.sync()
    off, r = [], []
    for b in range(3):
        k, v = s.want.values(s.table[b], c)
        want, p, _, _ = ko.attend(_np(q)[b * n:(b + 1) * n], k, v, hd ** -0.5)
        off.append(_np(out)[b * n:(b + 1) * n] != want.astype(np.float16).astype(np.float64))
        r.append((2.0 ** -4.5 / 3 ** 0.5) ** 3 * np.sqrt(np.einsum("nhc,chd->nhd", p ** 2, np.repeat(v, G, 1) ** 2)) / want)
    return np.mean(off), 2 * np.mean(r) * 2 ** 11


@pytest.mark.parametrize("G,hd,n", [(4, 128, 1), (8, 64, 1), (2, 128, 2), (16, 128, 1), (32, 64, 1)])
def test_attend_weights_keep_their_bits(torch, corun, G, hd, n):
    off, most = _share_not_nearest(torch, corun, G, hd, n, seed=G + hd)
    assert off <= most


# ---------------------------------------------------------------- append: layouts that are read value by value

N_NEW, START = [1, 2, 5, 16, 35, 1, 17, 3], [0, 7, 14, 0, 9, 48, 16, 100]


def _off_16(torch, t):
    """The same values in a layout whose heads do not start on 16 bytes."""
    big = torch.empty(*t.shape[:-1], t.shape[-1] + 1, dtype=t.dtype, device=t.device)
    big[..., 1:] = t
    return big[..., 1:]


def _append_case(torch, corun, hd, n_kv, G, dtype, seed):
    dt = getattr(torch, dtype)
    ctx = [a + b for a, b in zip(START, N_NEW)]
    ctx[1] = 0
    s = Setup(torch, corun, ctx, n_kv, hd, 16, seed=seed)
    T = sum(N_NEW)
    scale = 10.0 ** s.rng.uniform(-3, 3, (T, (G + 2) * n_kv, 1))
    x = torch.tensor(s.rng.standard_normal((T, (G + 2) * n_kv, hd)) * scale).clamp(-6e4, 6e4).to(dt).cuda()
    q, k, v = (t.contiguous() for t in x.split([G * n_kv, n_kv, n_kv], 1))
    pos = s.rng.integers(0, 100000, T).astype(np.int32)
    return s, ctx, q, k, v, pos, _i32(torch, np.concatenate([[0], np.cumsum(N_NEW)]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("hd,n_kv,G", [(128, 2, 3), (64, 3, 1)])
@pytest.mark.parametrize("rot,interleaved", [(6, False), (6, True), (20, False), (36, True), (36, False), (62, False), (64, True), (64, False), (0, False)])
@pytest.mark.parametrize("off", [False, True])
def test_append_value_by_value(torch, corun, dtype, hd, n_kv, G, rot, interleaved, off):
    """Rotated parts that are no whole pieces of 16 bytes and heads that do not start on 16 bytes, queries in place."""
    s, ctx, q, k, v, pos, cu = _append_case(torch, corun, hd, n_kv, G, dtype, seed=rot + hd)
    rope = corun.Rope(rot, theta=1e6, interleaved=interleaved) if rot else None
    # the same call on a copy of the cache through aligned tensors: the same bytes
    other = corun.Kv8Cache(s.cache.pages, n_kv, hd, 16, pool=s.cache.pool.clone(), exps=s.cache.exps.clone())
    args = dict(cu=cu, positions=_i32(torch, pos), rope=rope)
    q_want = other.append(k, v, _i32(torch, ctx), s.t_table, q=q, q_out=torch.full_like(q, 9.0), **args)
    if off:
        qi, ki, vi = (_off_16(torch, t) for t in (q, k, v))
    else:
        qi, ki, vi = q.clone(), k, v
    mass = torch.full((len(ctx), n_kv, s.max_blocks * 16), 3.0, device="cuda")
    assert s.cache.append(ki, vi, _i32(torch, ctx), s.t_table, q=qi, q_out=qi, mass=mass, **args) is qi
    live = torch.tensor(np.repeat(np.array(ctx) > 0, N_NEW), device="cuda")
    assert torch.equal(qi[live], q_want[live]) and torch.equal(qi[~live], q[~live])
    codes, exps = s.state()
    assert np.array_equal(codes, other.pool.view(torch.uint8).cpu().numpy()) and np.array_equal(exps, other.exps.cpu().numpy())
    # against 64 bits
    f, m = ko.frequencies(rot, theta=1e6) if rot else (np.zeros(0), 1.0)
    kr, qr = (ko.rotate(_np(t), pos, f, m, interleaved) for t in (k, q))
    bound = _eps(torch, q.dtype) * np.abs(qr) + 8 * 2.0 ** -24 * np.abs(_np(q)).max(-1, keepdims=True) + (2.0 ** -25 if dtype == "float16" else 0)
    alive = live.cpu().numpy()
    assert np.all((np.abs(_np(qi) - qr) <= bound)[alive])
    touched, at, first = np.zeros(codes.shape[0], bool), 0, s.codes
    for b, n in enumerate(N_NEW):
        if ctx[b] and n:
            kk, vv = kr[at:at + n], _np(v)[at:at + n]
            assert bool((mass[b, :, START[b]:ctx[b]] == 0).all()) and bool((mass[b, :, :START[b]] == 3).all()) and bool((mass[b, :, ctx[b]:] == 3).all())
            for jb in range(START[b] // 16, (ctx[b] - 1) // 16 + 1):
                pg, z0, z1 = s.table[b, jb], max(0, START[b] - jb * 16), min(16, ctx[b] - jb * 16)
                touched[pg] = True
                t0 = jb * 16 + z0 - START[b]
                for kind, x in ((0, kk), (1, vv)):
                    for h in range(n_kv):
                        new, e = x[t0:t0 + z1 - z0, h], int(exps[pg, kind, h])
                        slack = 8 * 2.0 ** -24 * np.abs(_np(k)[at + t0:at + t0 + z1 - z0, h]).max() if kind == 0 else 0.0
                        old = int(s.exps[pg, kind, h]) if z0 else ko.E_MIN
                        assert max(old, ko.exponent(max(np.abs(new).max() - slack, 0))) <= e <= max(old, ko.exponent(np.abs(new).max() + slack))
                        _check_values(codes[pg, kind, h, z0:z1], new / 2.0 ** e, None, slack / 2.0 ** e)
                        if z0:
                            moved = ko.encode(ko.decode(first[pg, kind, h, :z0]) * 2.0 ** (old - e)) if e > old else first[pg, kind, h, :z0]
                            assert np.array_equal(codes[pg, kind, h, :z0], moved)
        at += n
    assert np.array_equal(codes[~touched], s.codes[~touched]) and np.array_equal(exps[~touched], s.exps[~touched])


# ---------------------------------------------------------------- chunks behind long contexts

@pytest.mark.parametrize("n_kv,G,hd,block,dtype", [(2, 4, 128, 16, "bfloat16"), (1, 8, 64, 64, "float16"), (1, 5, 128, 32, "float16"), (2, 8, 64, 16, "bfloat16")])
@pytest.mark.parametrize("window", [0, 1500])
def test_chunks_behind_long_contexts(torch, corun, n_kv, G, hd, block, dtype, window):
    """Rows of more than 32 columns over 20 to 70 blocks of 128 tokens, scales that differ from page to page by up to 2^12, beside a row of one token."""
    ctx, n = [5000, 2600, 9000, 700], [50, 40, 9, 1]
    s = Setup(torch, corun, ctx, n_kv, hd, block, seed=G + hd)
    e = s.exps.astype(np.int32)
    e[:, 0] += s.rng.integers(-6, 1, e[:, 0].shape)
    e[:, 1] += s.rng.integers(-6, 7, e[:, 1].shape)
    s.want.exps = e
    s.cache.exps.copy_(torch.tensor(e.astype(np.int8)))
    T = sum(n)
    q = torch.tensor(s.rng.standard_normal((T, G * n_kv, hd)) * 0.3).to(getattr(torch, dtype)).cuda()
    out = torch.full((T + 1, G * n_kv, hd), 5.0, dtype=q.dtype, device="cuda")
    cu = _i32(torch, np.concatenate([[0], np.cumsum(n)]))
    att = corun.Kv8Attention(4, G * n_kv, n_kv, hd, s.max_blocks, block, tokens=T, max_new=50)
    att.run(q, s.cache, _i32(torch, ctx), s.t_table, hd ** -0.5, cu=cu, window=window, out=out[:T])
    att.sync()
    assert bool((out[T] == 5).all())
    _check_attend(torch, s, q, out, None, None, ctx, n, window, hd ** -0.5)
