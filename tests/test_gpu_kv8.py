"""Rotary positions, the 8-bit cache, attention over it and eviction from it against their 64-bit oracle.

Tolerances.  eps / 2 of a type is the rounding of one value.  Rotations: cos and sin are within 2^-24, two products and a
sum add 2^-24 each of |x1| + |x2|: 4 * 2^-24 (|x1| + |x2|) m in all.  Attention: the scores' sums of up to 128 products
in 32 bits are within 128 * 2^-24 of the sum A of the products' magnitudes, so a weight is within 2 * 2^-17 A of its
value; weights enter the product with values with 11 bits (2^-11 relative, and the sum of weights alike), which leaves
|out - exact| <= eps / 2 |exact| + (2 * 2^-11 + 2^-16 A) sum p |v|."""
import numpy as np
import pytest

from oracle import kv8_oracle as ko

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    return t


@pytest.fixture(scope="module")
def corun():
    from paper_2608_14376_b200 import corun

    return corun


def _np(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.cpu().numpy()


def _eps(torch, dt):
    return torch.finfo(dt).eps / 2


# ---------------------------------------------------------------- rotary positions

OPTIONS = [dict(), dict(interleaved=True), dict(theta=1e6, scaling="linear", factor=4.0), dict(theta=1e6, scaling="base", factor=8.0),
           dict(theta=1e6, scaling="parts", factor=32.0, original_context=4096), dict(scaling="parts", factor=4.0, original_context=256, low=2.0, high=16.0),
           dict(theta=5e5, scaling="bands", factor=8.0, original_context=8192, high=4.0, interleaved=True), dict(magnitude=0.5)]


@pytest.mark.parametrize("opt", OPTIONS, ids=str)
@pytest.mark.parametrize("T,heads,dim,rot,dtype,far", [(1, 40, 128, 128, "bfloat16", 5), (3, 1, 64, 64, "float16", 1 << 20), (37, 5, 128, 64, "float32", 131072),
                                                       (301, 3, 96, 48, "bfloat16", 4096), (9, 7, 80, 20, "float32", 70000), (5, 2, 10, 6, "float16", 99),
                                                       (2, 2, 256, 256, "float32", 3000000)])
def test_rope(torch, corun, opt, T, heads, dim, rot, dtype, far):
    if opt.get("scaling") == "parts" and rot == 6:
        opt = dict(opt, low=0.5)
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(T + dim)
    x = torch.randn(T, heads + 2, dim, generator=g).to(dt).cuda()[:, 1:heads + 1]
    pos = torch.randint(0, far, (T,), generator=g, dtype=torch.int32)
    rope = corun.Rope(rot, **opt)
    y = rope.apply(x, pos.cuda())
    f, m = ko.frequencies(rot, **opt)
    want = ko.rotate(_np(x), pos.numpy(), f, m, opt.get("interleaved", False))
    ax = np.abs(_np(x))
    i1, i2 = (slice(0, rot, 2), slice(1, rot, 2)) if opt.get("interleaved") else (slice(0, rot // 2), slice(rot // 2, rot))
    both = np.zeros_like(want)
    both[..., i1] = both[..., i2] = ax[..., i1] + ax[..., i2]
    tiny = 2.0 ** -25 if dtype == "float16" else 0.0            # half the smallest subnormal step
    assert np.all(np.abs(_np(y) - want) <= _eps(torch, dt) * np.abs(want) + 4 * 2.0 ** -24 * both * m + tiny)
    assert torch.equal(y[..., rot:], x[..., rot:])
    # in place, and through a layout that is read value by value: the same bits
    z = x.clone()
    assert rope.apply(z, pos.cuda(), out=z) is z and torch.equal(z, y)
    odd = torch.empty(T, heads, dim + 1, dtype=dt, device="cuda")[..., 1:]
    odd.copy_(x)
    assert torch.equal(rope.apply(odd, pos.cuda()), y)
    wide = torch.full((T, heads, dim + 3), 7.0, dtype=dt, device="cuda")
    rope.apply(x, pos.cuda(), out=wide[..., :dim])
    assert torch.equal(wide[..., :dim], y) and bool((wide[..., dim:] == 7).all())


def test_rope_negative_positions_undo(torch, corun):
    x = torch.randn(17, 4, 64, device="cuda")
    pos = torch.arange(17, dtype=torch.int32, device="cuda") * 1000
    rope = corun.Rope(64)
    back = rope.apply(rope.apply(x, pos), -pos)
    # two rotations, each within 4 * 2^-24 (|x1| + |x2|), the second one's input off by the first's error
    assert float((back - x).abs().max()) <= 12 * 2.0 ** -24 * 2 * float(x.abs().max())
    assert rope.apply(x[:0], pos[:0]).shape == (0, 4, 64)


# ---------------------------------------------------------------- the cache

class Setup:
    """A pool with pages dealt at random, rows with `ctx` tokens of old content (codes at random, NaN behind the rows' ends)."""

    def __init__(self, torch, corun, ctx, n_kv, hd, block, seed, spare_blocks=2, nan_behind=True):
        rng = np.random.default_rng(seed)
        self.rng, self.block, self.n_kv, self.hd = rng, block, n_kv, hd
        self.max_blocks = max(-(-max(c, 1) // block) for c in ctx) + spare_blocks
        pages = sum(-(-max(c, 1) // block) + spare_blocks for c in ctx) + 3
        order = list(rng.permutation(pages))
        self.table = np.zeros((len(ctx), self.max_blocks), np.int32)
        for b, c in enumerate(ctx):
            for i in range(-(-max(c, 1) // block) + spare_blocks):
                self.table[b, i] = order.pop()
        self.free = order
        self.codes = ko.encode(rng.standard_normal((pages, 2, n_kv, block, hd)) * 100)
        self.exps = rng.integers(-9, -4, (pages, 2, n_kv)).astype(np.int8)
        if nan_behind:
            used = np.zeros((pages, block), bool)
            for b, c in enumerate(ctx):
                for j in range(c):
                    used[self.table[b, j // block], j % block] = True
            self.codes = np.where(used[:, None, None, :, None], self.codes, 0x7F).astype(np.uint8)
        self.cache = corun.Kv8Cache(pages, n_kv, hd, block, pool=torch.tensor(self.codes).cuda().view(torch.float8_e4m3fn),
                                    exps=torch.tensor(self.exps).cuda())
        self.want = ko.Cache(self.codes, self.exps)
        self.t_table = torch.tensor(self.table).cuda()
        self.torch = torch

    def state(self):
        return self.cache.pool.view(self.torch.uint8).cpu().numpy(), self.cache.exps.cpu().numpy()


def _i32(torch, v):
    return torch.tensor(np.asarray(v, np.int32)).cuda()


def _check_values(got, want, exps, slack):
    """Stored codes against exact values (want, in units of the block): within half a step, where `slack` (same units) is how far
    the value itself may be off."""
    v = ko.decode(got)
    w = np.clip(want, -448, 448)
    step = np.maximum(2.0 ** -9, 2.0 ** (np.floor(np.log2(np.maximum(np.abs(w) + slack, 1e-30))) - 3))
    assert np.all(np.abs(v - w) <= step / 2 + slack)


@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("hd,n_kv,G,dtype", [(128, 8, 4, "bfloat16"), (64, 1, 1, "float16"), (128, 2, 3, "float32"), (64, 3, 8, "bfloat16")])
def test_append(torch, corun, block, hd, n_kv, G, dtype):
    dt = getattr(torch, dtype)
    n = [1, 0, 5, block, 2 * block + 3, 1, 17, 3]
    start = [0, 7, block - 2, 0, 9, 3 * block, block, 100]
    ctx = [s + m for s, m in zip(start, n)]
    ctx[1] = 0                                                  # a padding row
    s = Setup(torch, corun, [c for c in ctx], n_kv, hd, block, seed=hd + block)
    T = sum(n)
    rng = s.rng
    scale = 10.0 ** rng.uniform(-3, 3, (T + 2, n_kv + G * n_kv + n_kv, 1))      # pages whose scale grows and pages whose scale does not
    qkv = torch.tensor(rng.standard_normal((T + 2, G * n_kv + 2 * n_kv, hd)) * scale).clamp(-6e4, 6e4).to(dt).cuda()
    q, k, v = qkv.split([G * n_kv, n_kv, n_kv], 1)
    pos = rng.integers(0, 100000, T + 2).astype(np.int32)
    rot = hd // 2 if G == 3 else hd
    rope = corun.Rope(rot, theta=1e6, interleaved=G == 8)
    mass = torch.full((len(n), n_kv, s.max_blocks * block), 3.0, device="cuda")
    q_out = torch.full((T + 2, G * n_kv, hd), 9.0, dtype=dt, device="cuda")
    cu = _i32(torch, np.concatenate([[0], np.cumsum(n)]))
    ret = s.cache.append(k, v, _i32(torch, ctx), s.t_table, cu=cu, positions=_i32(torch, pos), rope=rope, q=q, q_out=q_out, mass=mass)
    assert ret is q_out
    codes, exps = s.state()
    f, m = ko.frequencies(rot, theta=1e6)
    kr = ko.rotate(_np(k), pos, f, m, G == 8)
    kr32 = kr.astype(np.float32).astype(np.float64)
    at = 0
    touched = np.zeros(codes.shape[0], bool)
    for b in range(len(n)):
        if ctx[b] and n[b]:
            s.want.append(s.table[b], start[b], kr32[at:at + n[b]], _np(v)[at:at + n[b]])
            touched[s.table[b, start[b] // block:(ctx[b] - 1) // block + 1]] = True
        at += n[b]
    assert np.array_equal(exps, s.want.exps)
    assert np.array_equal(codes[:, 1], s.want.codes[:, 1])      # values: to the last bit
    assert np.array_equal(codes[~touched], s.codes[~touched])
    at = 0
    for b in range(len(n)):
        for i in range(n[b] if ctx[b] else 0):
            j = start[b] + i
            pg = s.table[b, j // block]
            e = 2.0 ** exps[pg, 0].astype(np.float64)[:, None]
            x = np.abs(_np(k)[at + i])
            _check_values(codes[pg, 0, :, j % block], kr[at + i] / e, exps[pg, 0], 4 * 2.0 ** -24 * 2 * x.max(-1, keepdims=True) / e)
        if ctx[b] and n[b]:                                     # old keys of the first page moved with its scale
            pg, z = s.table[b, start[b] // block], start[b] % block
            assert np.array_equal(codes[pg, 0, :, :z], s.want.codes[pg, 0, :, :z])
            assert bool((mass[b, :, start[b]:ctx[b]] == 0).all())
        assert bool((mass[b, :, :start[b] if ctx[b] else ctx[b]] == 3).all()) and bool((mass[b, :, ctx[b]:] == 3).all())
        at += n[b]
    want_q = ko.rotate(_np(q), pos, f, m, G == 8)
    bound = _eps(torch, dt) * np.abs(want_q) + 8 * 2.0 ** -24 * np.abs(_np(q)).max(-1, keepdims=True) + (2.0 ** -25 if dtype == "float16" else 0)
    live = np.concatenate([np.full(m_, bool(c)) for m_, c in zip(n, ctx)] + [np.zeros(2, bool)])
    got_q = _np(q_out)
    assert np.all((np.abs(got_q - want_q) <= bound)[live]) and np.all(got_q[~live] == 9)      # tokens of no row are left as they were


def test_append_step_by_step_and_in_place(torch, corun):
    """One token at a time (no cu) into the same pages: as one call would have stored them, but for subnormals; queries in place."""
    B, n_kv, hd, steps = 3, 2, 128, 20
    s = Setup(torch, corun, [0, 0, 0], n_kv, hd, 16, seed=4)
    x = torch.tensor(s.rng.standard_normal((steps, B, 3 * n_kv, hd))).to(torch.bfloat16).cuda()
    for i in range(steps):
        q, k, v = (t.contiguous() for t in x[i].split([n_kv] * 3, 1))
        before = q.clone()
        assert s.cache.append(k, v, _i32(torch, [i + 1, 0, i + 1]), s.t_table, q=q, q_out=q) is q and torch.equal(q, before)
    codes, exps = s.state()
    for b in (0, 2):
        s.want.append(s.table[b], 0, *(_np(x[:, b, j * n_kv:(j + 1) * n_kv]) for j in (1, 2)))
    assert np.array_equal(exps, s.want.exps)
    for b in (0, 2):
        k, v = s.want.values(s.table[b], steps)
        got = ko.Cache(codes, exps)
        for w, g in zip((k, v), got.values(s.table[b], steps)):
            e = exps[s.table[b][np.arange(steps) // 16], 0]
            assert np.mean(w != g) < 0.01                       # rounded twice among the subnormals
            assert np.abs(w - g).max() <= 2.0 ** -9 * 2.0 ** float(exps.max())


def test_append_specials_and_bad_pages(torch, corun):
    """NaN stay, infinities are cut at the top of the block, pages outside the pool are not written."""
    s = Setup(torch, corun, [3, 2], 1, 64, 16, seed=5)
    k = torch.randn(2, 1, 64, device="cuda")
    k[0, 0, 3], k[0, 0, 4], k[0, 0, 5] = float("nan"), float("inf"), -float("inf")
    v = torch.zeros(2, 1, 64, device="cuda")
    table = s.t_table.clone()
    table[1, 0] = s.codes.shape[0]                              # beyond the pool
    s.cache.append(k, v, _i32(torch, [1, 2]), table)
    codes, exps = s.state()
    pg = s.table[0, 0]
    assert exps[pg, 0, 0] == 31 and exps[pg, 1, 0] == -32
    row = codes[pg, 0, 0, 0]
    assert row[3] & 0x7F == 0x7F and row[4] == 0x7E and row[5] == 0xFE
    assert not codes[pg, 1, 0, 0].any()
    others = np.ones(len(codes), bool)
    others[pg] = False
    assert np.array_equal(codes[others], s.codes[others]) and np.array_equal(exps[others], s.exps[others])
    table[1, 0] = -1
    s.cache.append(k, v, _i32(torch, [1, 2]), table)
    assert np.array_equal(s.state()[0][others], s.codes[others])
    # rows that are left out: more new tokens than cached ones, beyond the table, tokens outside the call
    before = s.state()
    for ctx, cu in (([1, 1], [0, 2, 2]), ([s.max_blocks * 16 + 1, 0], [0, 1, 1]), ([3, 2], [-1, 0, 3]), ([3, 2], [2, 1, 0])):
        s.cache.append(k, v, _i32(torch, ctx), s.t_table, cu=_i32(torch, cu))
    after = s.state()
    assert np.array_equal(before[0], after[0]) and np.array_equal(before[1], after[1])


# ---------------------------------------------------------------- attention

def _attend_case(torch, corun, ctx, n, n_kv, G, hd, block, dtype, window=0, mass=False, seed=0, q_std=1.5, table_fn=None):
    s = Setup(torch, corun, ctx, n_kv, hd, block, seed)
    dt = getattr(torch, dtype)
    T = sum(n)
    q = torch.tensor(s.rng.standard_normal((T, G * n_kv, hd)) * q_std * 0.05).to(dt).cuda()
    out = torch.full((T + 1, G * n_kv, hd), 5.0, dtype=dt, device="cuda")[:T]
    cu = None if n == [1] * len(n) else _i32(torch, np.concatenate([[0], np.cumsum(n)]))
    m = torch.rand(len(ctx), n_kv, s.max_blocks * block, device="cuda") if mass else None
    m0 = _np(m) if mass else None
    att = corun.Kv8Attention(len(ctx), G * n_kv, n_kv, hd, s.max_blocks, block, tokens=T, max_new=max(n))
    scale = hd ** -0.5
    att.run(q, s.cache, _i32(torch, ctx), s.t_table, scale, cu=cu, window=window, mass=m, out=out)
    att.sync()
    return s, q, out, m, m0, scale


def _check_attend(torch, s, q, out, m, m0, ctx, n, window, scale):
    got, at = _np(out), 0
    for b, (c, k_new) in enumerate(zip(ctx, n)):
        mine = got[at:at + k_new]
        if c == 0:
            assert np.all(mine == 5.0)                          # a padding row is left alone
        elif k_new:
            k, v = s.want.values(s.table[b], c)
            want, p, a, pv = ko.attend(_np(q)[at:at + k_new], k, v, scale, window)
            bound = _eps(torch, q.dtype) * np.abs(want) + (2 * 2.0 ** -11 + 2.0 ** -16 * a[..., None]) * pv
            if q.dtype == torch.float16:
                bound = bound + 2.0 ** -25
            assert np.all(np.abs(mine - want) <= bound), (b, float((np.abs(mine - want) / bound).max()))
            if m is not None:
                g = np.einsum("nhc->hc", p).reshape(s.n_kv, -1, c).sum(1)
                tol = np.einsum("nhc,nh->hc", p, 2.0 ** -16 * a + 2.0 ** -21).reshape(s.n_kv, -1, c).sum(1) + 2.0 ** -22 * (m0[b, :, :c] + g)
                assert np.all(np.abs(_np(m)[b, :, :c] - m0[b, :, :c] - g) <= tol)
        if m is not None:
            assert np.array_equal(_np(m)[b, :, c:], m0[b, :, c:])
        at += k_new


CTX = [0, 1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 300, 513, 1030]


@pytest.mark.parametrize("n_kv,G,hd,block,dtype", [(8, 4, 128, 16, "bfloat16"), (2, 1, 64, 16, "float16"), (1, 8, 128, 64, "bfloat16"), (3, 2, 64, 32, "bfloat16"),
                                                   (2, 3, 128, 16, "float16"), (1, 16, 128, 32, "float16"), (1, 32, 64, 64, "bfloat16"), (2, 5, 128, 16, "bfloat16"),
                                                   (1, 9, 64, 16, "float16")])
@pytest.mark.parametrize("window,mass", [(0, False), (0, True), (130, True)])
def test_attend_one_token(torch, corun, n_kv, G, hd, block, dtype, window, mass):
    n = [1] * len(CTX)
    r = _attend_case(torch, corun, CTX, n, n_kv, G, hd, block, dtype, window, mass, seed=G + hd)
    _check_attend(torch, r[0], r[1], r[2], r[3], r[4], CTX, n, window, r[5])


@pytest.mark.parametrize("n_kv,G,hd,block,dtype", [(2, 4, 128, 16, "bfloat16"), (1, 1, 64, 16, "float16"), (2, 8, 128, 64, "float16"), (1, 3, 64, 32, "bfloat16"),
                                                   (1, 32, 128, 16, "bfloat16")])
@pytest.mark.parametrize("window", [0, 40])
def test_attend_ragged_tokens(torch, corun, n_kv, G, hd, block, dtype, window):
    ctx = [1, 0, 33, 128, 129, 300, 700, 20]
    n = [1, 2, 33, 7, 129, 1, 60, 0]
    r = _attend_case(torch, corun, ctx, n, n_kv, G, hd, block, dtype, window, seed=3)
    _check_attend(torch, r[0], r[1], r[2], r[3], r[4], ctx, n, window, r[5])


@pytest.mark.parametrize("n_kv,G", [(2, 4), (1, 8), (4, 1)])
def test_attend_few_tokens_with_weights(torch, corun, n_kv, G):
    ctx, n = [5, 140, 700, 9], [3, 4, 2, 1]
    r = _attend_case(torch, corun, ctx, n, n_kv, G, 128, 16, "bfloat16", 0, True, seed=9)
    _check_attend(torch, r[0], r[1], r[2], r[3], r[4], ctx, n, 0, r[5])


def test_attend_peaked_and_uneven_scales(torch, corun):
    """Sharp softmax, pages whose values' scales differ by 2^20: the tokens that count keep their precision."""
    for spread in (3, 20):
        s = Setup(torch, corun, [400, 129], 2, 128, 16, seed=spread)
        e = s.exps.astype(np.int32)
        e[:, 1] += s.rng.integers(-spread, spread + 1, e[:, 1].shape)
        s.want.exps = np.clip(e, -32, 31)
        s.cache.exps.copy_(torch.tensor(s.want.exps.astype(np.int8)))
        q = torch.tensor(s.rng.standard_normal((2, 8, 128)) * 0.6).to(torch.bfloat16).cuda()
        att = corun.Kv8Attention(2, 8, 2, 128, s.max_blocks, 16)
        out = torch.full((2, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        att.run(q, s.cache, _i32(torch, [400, 129]), s.t_table, 128 ** -0.5, out=out)
        att.sync()
        _check_attend(torch, s, q, out, None, None, [400, 129], [1, 1], 0, 128 ** -0.5)


def test_attend_long_and_rows_are_independent(torch, corun):
    """A row's bytes are the same alone, among other rows, in another place and with its pages elsewhere; twice the same."""
    ctx = [5000, 77, 40000, 3]
    s = Setup(torch, corun, ctx, 2, 128, 16, seed=1)
    q = torch.tensor(s.rng.standard_normal((4, 8, 128)) * 0.1).to(torch.bfloat16).cuda()
    run = lambda t, c, qq, cache=None: corun.Kv8Attention(len(c), 8, 2, 128, t.shape[1], 16).run(qq, cache or s.cache, _i32(torch, c), t.contiguous(), 0.088)
    base = run(s.t_table, ctx, q)
    assert torch.equal(base, run(s.t_table, ctx, q))
    _check_attend(torch, s, q, base, None, None, ctx, [1] * 4, 0, np.float32(0.088).astype(np.float64))
    perm = [2, 0, 3]
    assert torch.equal(run(s.t_table[perm], [ctx[i] for i in perm], q[perm].contiguous()), base[perm])
    shuffle = torch.randperm(s.cache.pages, device="cuda")
    where = torch.empty_like(shuffle)
    where[shuffle] = torch.arange(s.cache.pages, device="cuda")
    moved = corun.Kv8Cache(s.cache.pages, 2, 128, 16, pool=s.cache.pool.view(torch.uint8)[shuffle].view(torch.float8_e4m3fn), exps=s.cache.exps[shuffle])
    assert torch.equal(run(where[s.t_table.long()].int(), ctx, q, moved), base)
    # one token among rows with many: the same bytes again
    n = [1, 40, 1, 2]
    qq = torch.zeros(44, 8, 128, dtype=torch.bfloat16, device="cuda")
    qq[0], qq[41] = q[0], q[2]
    att = corun.Kv8Attention(4, 8, 2, 128, s.max_blocks, 16, tokens=44, max_new=40)
    out = att.run(qq, s.cache, _i32(torch, ctx), s.t_table, 0.088, cu=_i32(torch, [0, 1, 41, 42, 44]))
    assert torch.equal(out[0], base[0]) and torch.equal(out[41], base[2])


def test_attend_left_out_rows_and_bad_pages(torch, corun):
    s = Setup(torch, corun, [40, 40, 2], 1, 64, 16, seed=2)
    q = torch.randn(3, 2, 64, device="cuda").to(torch.float16)
    att = corun.Kv8Attention(3, 2, 1, 64, s.max_blocks, 16, tokens=6, max_new=4)
    out = torch.full((3, 2, 64), 5.0, dtype=torch.float16, device="cuda")
    # beyond the table; more new tokens than cached ones (its first query sees nothing); empty
    att.run(q, s.cache, _i32(torch, [s.max_blocks * 16 + 1, 1, 0]), s.t_table, 0.125, cu=_i32(torch, [0, 1, 3, 3]), out=out)
    att.sync()
    assert bool((out[0] == 5).all()) and bool((out[1] == 0).all())
    v = s.want.values(s.table[1], 1)[1][0, 0]
    assert np.all(np.abs(_np(out)[2] - v) <= _eps(torch, torch.float16) * np.abs(v) + 2 * 2.0 ** -11 * np.abs(v))
    # a page outside the pool stands for zeros, whatever its number
    for bad in (s.cache.pages, -1, 2 ** 31 - 1, -2 ** 31):
        t = s.t_table.clone()
        t[0, 1] = bad
        out = corun.Kv8Attention(3, 2, 1, 64, s.max_blocks, 16).run(q, s.cache, _i32(torch, [40, 0, 0]), t, 0.125)
        k, v = s.want.values(s.table[0], 40)
        k[16:32] = v[16:32] = 0
        want, _, a, pv = ko.attend(_np(q)[:1], k, v, 0.125)
        assert np.all(np.abs(_np(out)[:1] - want) <= _eps(torch, torch.float16) * np.abs(want) + (2 * 2.0 ** -11 + 2.0 ** -16 * a[..., None]) * pv + 2.0 ** -25)


def test_attend_strided_queries_graphs_and_streams(torch, corun):
    ctx = [300, 17, 1000]
    s = Setup(torch, corun, ctx, 2, 128, 16, seed=7)
    big = torch.randn(3, 12, 128, device="cuda").to(torch.bfloat16)
    q = big[:, 2:10]
    att = corun.Kv8Attention(3, 8, 2, 128, s.max_blocks, 16)
    t_ctx = _i32(torch, ctx)
    want = att.run(q, s.cache, t_ctx, s.t_table, 0.1)
    wide = torch.zeros(3, 9, 128, dtype=torch.bfloat16, device="cuda")
    att.run(q, s.cache, t_ctx, s.t_table, 0.1, out=wide[:, 1:])
    assert torch.equal(wide[:, 1:], want) and not bool(wide[:, 0].any())
    # two calls captured into two graphs, replayed on two streams at once, with other lengths than at capture
    outs, graphs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for st in streams:
        g, o = torch.cuda.CUDAGraph(), torch.zeros_like(want)
        with torch.cuda.graph(g, stream=st):
            att.run(q, s.cache, t_ctx, s.t_table, 0.1, out=o)
        graphs.append(g)
        outs.append(o)
    t_ctx.copy_(_i32(torch, [1000 if i == 2 else 10 for i in range(3)]))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    again = corun.Kv8Attention(3, 8, 2, 128, s.max_blocks, 16).run(q, s.cache, t_ctx, s.t_table, 0.1)
    for o in outs:
        assert torch.equal(o, again)
    assert torch.equal(again[2], want[2])
    # eager calls on another stream than the tensors' own
    with torch.cuda.stream(streams[0]):
        o = att.run(q, s.cache, t_ctx, s.t_table, 0.1)
        att.sync()
    assert torch.equal(o, again)


# ---------------------------------------------------------------- eviction

@pytest.mark.parametrize("block,hd,n_kv", [(16, 128, 8), (32, 64, 2), (64, 128, 1)])
def test_evict(torch, corun, block, hd, n_kv):
    ctx = [700, 40, 0, 65, 2000, 64, 333, 70]
    keep = [200, 64, 10, 64, 3, 64, 0, 69]
    max_keep, sinks, recent = 210, 3, 30
    s = Setup(torch, corun, ctx, n_kv, hd, block, seed=block)
    s.exps = (s.exps + s.rng.integers(-6, 7, s.exps.shape)).astype(np.int8)       # scales that differ from block to block
    s.cache.exps.copy_(torch.tensor(s.exps))
    s.want = ko.Cache(s.codes, s.exps)
    reach = s.max_blocks * block
    m = s.rng.random((len(ctx), n_kv, reach)).astype(np.float32) ** 4
    m[:, :, ::3] = 0.25                                          # ties
    m[0, 0, 5:9] = np.nan
    m[4, :, 7:1000] = 0.0
    m[4, :, 100:200] = -0.0
    m[3] = 1.0
    mass = torch.tensor(m).cuda()
    kept, new_ctx = s.cache.evict(_i32(torch, ctx), s.t_table, mass, _i32(torch, keep), max_keep, sinks=sinks, recent=recent)
    kept, new_ctx = kept.cpu().numpy(), new_ctx.cpu().numpy()
    codes, exps = s.state()
    w = m.copy()
    for b, c in enumerate(ctx):
        k = min(max(keep[b], sinks + recent), max_keep) if keep[b] > 0 else 0
        if 0 < k < c:
            src = s.want.evict(s.table[b], c, w[b], k, sinks, recent)
            assert np.array_equal(kept[b, :, :k], src) and np.all(kept[b, :, k:] == -1) and new_ctx[b] == k
        else:
            assert np.all(kept[b] == -1) and new_ctx[b] == c
    assert np.array_equal(exps, s.want.exps)
    got, want = codes.copy(), s.want.codes.copy()
    for x in (got, want):                                        # -0 and what lies behind a row's new end are nobody's
        x[x == 0x80] = 0
    for b, c in enumerate(ctx):
        k = min(new_ctx[b], c)
        if k < c:
            for j in range(k, c):
                pg = s.table[b, j // block]
                got[pg, :, :, j % block] = want[pg, :, :, j % block] = 0
    assert np.array_equal(got, want)
    assert np.array_equal(mass.cpu().numpy(), w, equal_nan=True)


def test_evict_long_in_place_lengths_and_bad_pages(torch, corun):
    ctx = [30000, 900]
    s = Setup(torch, corun, ctx, 1, 64, 16, seed=6)
    m = s.rng.random((2, 1, s.max_blocks * 16)).astype(np.float32)
    mass, t = torch.tensor(m).cuda(), _i32(torch, ctx)
    table = s.t_table.clone()
    table[1, 3] = s.cache.pages                                  # a row with a bad page stays as it is
    kept, new_ctx = s.cache.evict(t, table, mass, _i32(torch, [20001, 100]), 20001, sinks=0, recent=0, new_ctx=t)
    assert new_ctx is t and t.tolist() == [20001, 900]
    src = s.want.evict(s.table[0], 30000, m[0], 20001, 0, 0)
    assert np.array_equal(kept[0].cpu().numpy(), src) and bool((kept[1] == -1).all())
    codes, exps = s.state()
    got = ko.Cache(codes, exps)
    for a, b in zip(got.values(s.table[0], 20001), s.want.values(s.table[0], 20001)):
        assert np.array_equal(a, b)
    for a, b in zip(got.values(s.table[1], 900), s.want.values(s.table[1], 900)):
        assert np.array_equal(a, b)


def test_evict_more_tokens_than_shared_memory_holds(torch, corun):
    ctx = [50001, 300]
    s = Setup(torch, corun, ctx, 1, 64, 64, seed=12)
    m = (s.rng.random((2, 1, s.max_blocks * 64)) ** 2).astype(np.float32)
    m[:, :, ::5] = 0.5
    mass = torch.tensor(m).cuda()
    kept, new_ctx = s.cache.evict(_i32(torch, ctx), s.t_table, mass, _i32(torch, [9000, 9000]), 9000, sinks=1, recent=7)
    assert new_ctx.tolist() == [9000, 300] and bool((kept[1] == -1).all())
    src = s.want.evict(s.table[0], 50001, m[0], 9000, 1, 7)
    assert np.array_equal(kept[0].cpu().numpy(), src) and np.array_equal(mass.cpu().numpy(), m)
    got = ko.Cache(*s.state())
    for a, b in zip(got.values(s.table[0], 9000), s.want.values(s.table[0], 9000)):
        assert np.array_equal(a, b)


def test_many_rows_are_what_few_rows_are(torch, corun):
    """300 rows in one call, empty ones among them: the bytes of six calls of 50."""
    rng = np.random.default_rng(3)
    ctx = [int(c) if c > 20 else 0 for c in rng.integers(0, 400, 300)]
    s = Setup(torch, corun, [max(c, 1) for c in ctx], 2, 64, 16, seed=13)
    other = corun.Kv8Cache(s.cache.pages, 2, 64, 16, pool=s.cache.pool.clone(), exps=s.cache.exps.clone())
    mk = lambda h: torch.tensor(rng.standard_normal((300, h, 64))).to(torch.float16).cuda()
    q, k, v, pos = mk(6), mk(2), mk(2), _i32(torch, rng.integers(0, 9999, 300))
    rope, t_ctx = corun.Rope(64), _i32(torch, ctx)
    q_all = s.cache.append(k, v, t_ctx, s.t_table, positions=pos, rope=rope, q=q, q_out=torch.zeros_like(q))
    out = corun.Kv8Attention(300, 6, 2, 64, s.max_blocks, 16).run(q_all, s.cache, t_ctx, s.t_table, 0.02)
    att = corun.Kv8Attention(50, 6, 2, 64, s.max_blocks, 16)
    for i in range(0, 300, 50):
        part = slice(i, i + 50)
        qp = other.append(k[part], v[part], t_ctx[part], s.t_table[part], positions=pos[part], rope=rope, q=q[part], q_out=torch.zeros_like(q[part]))
        o = att.run(qp, other, t_ctx[part], s.t_table[part], 0.02)
        att.sync()
        assert torch.equal(q_all[part], qp) and torch.equal(out[part], o)
    assert torch.equal(s.cache.pool.view(torch.uint8), other.pool.view(torch.uint8)) and torch.equal(s.cache.exps, other.exps)


# ---------------------------------------------------------------- together

def test_decode_with_eviction(torch, corun):
    """A prompt's chunk, decode steps that accumulate weights, an eviction, more steps: against the same program in 64 bits whose
    cache holds the same 8-bit values."""
    B, n_kv, G, hd, block = 3, 2, 4, 128, 16
    prompt = [70, 5, 33]
    s = Setup(torch, corun, [0] * B, n_kv, hd, block, seed=8, spare_blocks=8)
    rope = corun.Rope(hd, theta=1e6, scaling="parts", factor=4.0, original_context=64)
    scale = hd ** -0.5
    mass = torch.full((B, n_kv, s.max_blocks * block), 11.0, device="cuda")
    total = np.zeros((B, n_kv, s.max_blocks * block))
    ctx, pos = np.array(prompt), np.array(prompt)
    cu = np.concatenate([[0], np.cumsum(prompt)])
    T = cu[-1]
    make = lambda T: [t.contiguous() for t in torch.tensor(s.rng.standard_normal((T, (G + 2) * n_kv, hd))).to(torch.bfloat16).cuda().split([G * n_kv, n_kv, n_kv], 1)]
    q, k, v = make(T)
    p0 = np.concatenate([np.arange(n) for n in prompt])
    s.cache.append(k, v, _i32(torch, ctx), s.t_table, cu=_i32(torch, cu), positions=_i32(torch, p0), rope=rope, q=q, q_out=q, mass=mass)
    out = corun.Kv8Attention(B, G * n_kv, n_kv, hd, s.max_blocks, block, tokens=int(T), max_new=70).run(q, s.cache, _i32(torch, ctx), s.t_table, scale, cu=_i32(torch, cu))
    codes, exps = s.state()
    s.want = ko.Cache(codes, exps)
    _check_attend(torch, s, q, out, None, None, prompt, prompt, 0, scale)
    att = corun.Kv8Attention(B, G * n_kv, n_kv, hd, s.max_blocks, block)
    slack = np.zeros_like(total)
    for step in range(30):
        if step == 15:
            before = s.state()
            t_ctx = _i32(torch, ctx)
            w = _np(mass)
            kept, t_new = s.cache.evict(t_ctx, s.t_table, mass, _i32(torch, [40] * B), 40, sinks=2, recent=10)
            s.want = ko.Cache(*before)
            for b in range(B):
                if ctx[b] > 40:
                    ww = w[b].astype(np.float32)
                    src = s.want.evict(s.table[b], ctx[b], ww, 40, 2, 10)
                    assert np.array_equal(kept[b].cpu().numpy(), src)
                    for h in range(n_kv):
                        total[b, h, :40] = total[b, h, src[h]]
                        slack[b, h, :40] = slack[b, h, src[h]]
            now = s.state()
            assert np.array_equal(now[1], s.want.exps)
            ctx = np.minimum(ctx, 40)
            assert t_new.tolist() == ctx.tolist()
        ctx, pos = ctx + 1, pos + 1
        q, k, v = make(B)
        s.cache.append(k, v, _i32(torch, ctx), s.t_table, positions=_i32(torch, pos - 1), rope=rope, q=q, q_out=q, mass=mass)
        out = att.run(q, s.cache, _i32(torch, ctx), s.t_table, scale, mass=mass)
        s.want = ko.Cache(*s.state())
        _check_attend(torch, s, q, out, None, None, list(ctx), [1] * B, 0, scale)
        for b in range(B):
            kk, vv = s.want.values(s.table[b], ctx[b])
            _, p, a, _ = ko.attend(_np(q)[b:b + 1], kk, vv, scale)
            total[b, :, ctx[b] - 1], slack[b, :, ctx[b] - 1] = 0, 0
            total[b, :, :ctx[b]] += p[0].reshape(n_kv, G, -1).sum(1)
            slack[b, :, :ctx[b]] += (p[0] * (2.0 ** -16 * a[0][:, None] + 2.0 ** -21)).reshape(n_kv, G, -1).sum(1) + 2.0 ** -22 * total[b, :, :ctx[b]]
    for b in range(B):                                           # the prompt's tokens began at 0: append made them so
        assert np.all(np.abs(_np(mass)[b, :, :ctx[b]] - total[b, :, :ctx[b]]) <= slack[b, :, :ctx[b]])


@pytest.mark.parametrize("n_kv,G,hd,dtype", [(2, 8, 128, "float16"), (1, 8, 64, "float16"), (2, 4, 128, "bfloat16"), (1, 12, 128, "float16")])
def test_steps_replayed_from_a_graph(torch, corun, n_kv, G, hd, dtype):
    """Append and attention one behind the other in one captured graph, replayed with new inputs and lengths: the bytes of separate
    calls with a wait between them."""
    dt, B, block = getattr(torch, dtype), 3, 16
    s = Setup(torch, corun, [200, 31, 0], n_kv, hd, block, seed=G, spare_blocks=4)
    other = corun.Kv8Cache(s.cache.pages, n_kv, hd, block, pool=s.cache.pool.clone(), exps=s.cache.exps.clone())
    rope = corun.Rope(hd)
    att = corun.Kv8Attention(B, G * n_kv, n_kv, hd, s.max_blocks, block)
    mk = lambda h: torch.zeros(B, h, hd, dtype=dt, device="cuda")
    q, k, v, q_out, out = mk(G * n_kv), mk(n_kv), mk(n_kv), mk(G * n_kv), mk(G * n_kv)
    ctx, pos = _i32(torch, [200, 31, 0]), _i32(torch, [0, 0, 0])
    mass, mass2 = (torch.zeros(B, n_kv, s.max_blocks * block, device="cuda") for _ in range(2))

    def step(cache, mass, o, qo):
        cache.append(k, v, ctx, s.t_table, positions=pos, rope=rope, q=q, q_out=qo, mass=mass)
        return att.run(qo, cache, ctx, s.t_table, 0.05, mass=mass, out=o)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(s.cache, mass, out, q_out)
    for i in range(20):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda") * (4.0 ** (i % 4)))
        ctx += (ctx > 0).int()
        pos += 1
        g.replay()
        o2, q2 = torch.zeros_like(out), torch.zeros_like(q_out)
        torch.cuda.synchronize()
        other.append(k, v, ctx, s.t_table, positions=pos, rope=rope, q=q, q_out=q2, mass=mass2)
        torch.cuda.synchronize()
        att.run(q2, other, ctx, s.t_table, 0.05, mass=mass2, out=o2)
        att.sync()
        assert torch.equal(out[:2], o2[:2]) and torch.equal(q_out[:2], q2[:2]) and torch.equal(mass, mass2)
        assert torch.equal(s.cache.exps, other.exps)
    assert torch.equal(s.cache.pool.view(torch.uint8), other.pool.view(torch.uint8))
    _check_attend(torch, Sub(s), q_out[:2], out[:2], None, None, ctx.tolist()[:2], [1, 1], 0, float(np.float32(0.05)))


class Sub:
    """The cache as it is now, for ``_check_attend``."""

    def __init__(self, s):
        self.table, self.n_kv, self.want = s.table, s.n_kv, ko.Cache(*s.state())
