"""The 64-bit oracle of the 8-bit cache against torch's own e4m3 type and against small cases written out by hand; and the
refusals of the entry points, which need no GPU (every one comes before any CUDA call)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as ko


def test_codes_agree_with_torch():
    c = np.arange(256, dtype=np.uint8)
    t = torch.tensor(c).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ko.decode(c), t, equal_nan=True)
    rng = np.random.default_rng(0)
    # ordinary values, all midpoints between neighbours (ties), subnormals
    mid = (ko.TABLE[:126] + ko.TABLE[1:127]) / 2
    x = np.concatenate([rng.standard_normal(4000) * 10.0 ** rng.uniform(-4, 2.6, 4000), mid, -mid, ko.TABLE[:127], [0.0, -0.0, 448.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ko.encode(x), want)


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.5, 1), (896.0, 1), (224.0, -1), (1.75, -8), (1.0, -8), (1.7500001, -7), (0.0, -32),
                                    (1e-30, -32), (1e30, 31), (np.inf, 31)])
def test_exponents(amax, e):
    assert ko.exponent(amax) == e


def test_growing_page_keeps_old_values():
    codes = np.zeros((2, 2, 1, 16, 64), np.uint8)
    c = ko.Cache(codes, np.zeros((2, 2, 1), np.int8))
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 1, 64))
    c.append([1], 0, x[:3], x[:3])
    first = c.values([1], 3)[0]
    c.append([1], 3, 1000 * x[3:], x[3:])
    assert c.exps[1, 0, 0] > c.exps[1, 1, 0]
    now = c.values([1], 3)[0]
    step = 2.0 ** (c.exps[1, 0, 0] - 9)                      # the smallest step of the grown block
    assert np.all(np.abs(now - first) <= step / 2)


@pytest.fixture(scope="module")
def lib():
    from paper_2608_14376_b200 import build, corun

    build.build()
    return corun.lib()


BASE = 0x7F0000001000                                         # never dereferenced: the checks come first


def _parts():
    from paper_2608_14376_b200 import corun

    cache = corun.Kv8CacheArgs(BASE, BASE + 0x100000, 100, 16, 8, 128)
    rows = corun.Kv8Rows(BASE, 8, BASE, None, 4, 4)
    x = corun.Heads(BASE, 1024, 128)
    return corun, cache, rows, x


def test_rope_refusals(lib):
    from paper_2608_14376_b200 import corun

    def make(**kw):
        c = dict(rot_dim=64, interleaved=0, scaling=0, original_context=0, theta=1e4, factor=1.0, low=1.0, high=4.0, magnitude=0.0)
        c.update(kw)
        h = C.c_void_p()
        rc = lib.corun_rope_create(C.byref(corun.RopeConfig(**c)), C.byref(h))
        return rc, h

    for bad in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=258), dict(theta=0.0), dict(theta=float("nan")), dict(theta=float("inf")),
                dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")),
                dict(scaling=2, rot_dim=2, factor=2.0), dict(scaling=3, factor=2.0), dict(scaling=4, factor=2.0, original_context=10, low=4.0),
                dict(scaling=3, factor=2.0, original_context=10, theta=0.5), dict(magnitude=-1.0), dict(magnitude=float("inf"))):
        assert make(**bad)[0] == corun.EINVAL, bad
    assert lib.corun_rope_create(None, None) == corun.EINVAL
    rc, r = make()
    assert rc == corun.OK
    x = corun.Heads(BASE, 1024, 128)
    ok = [r, C.byref(x), C.byref(x), 1, BASE, 0, 8, 128, None]   # T = 0: nothing to launch
    assert lib.corun_rope_apply(*ok) == corun.OK
    for at, v in ((0, None), (1, None), (2, None), (3, 3), (3, -1), (4, None), (4, BASE + 2), (5, -1), (6, 0), (7, 63), (7, 1025)):
        a = list(ok)
        a[at] = v
        assert lib.corun_rope_apply(*a) == corun.EINVAL, (at, v)
    other = corun.Heads(BASE, 2048, 128)                          # in place with other strides
    assert lib.corun_rope_apply(r, C.byref(x), C.byref(other), 1, BASE, 0, 8, 128, None) == corun.EINVAL
    assert lib.corun_rope_apply(r, C.byref(corun.Heads(BASE + 1, 1, 1)), C.byref(x), 1, BASE, 0, 8, 128, None) == corun.EINVAL
    lib.corun_rope_destroy(r)
    lib.corun_rope_destroy(None)
    with pytest.raises(ValueError):
        corun.Rope(64, scaling="wide")
    with pytest.raises(corun.CorunError):
        corun.Rope(63)


@pytest.mark.parametrize("field,value", [("pool", None), ("exps", None), ("pool", BASE + 8), ("pages", 0), ("pages", 2**31), ("block", 8),
                                         ("block", 48), ("n_kv", 0), ("head_dim", 96), ("pages", 2**24)])
def test_bad_caches_are_refused_everywhere(lib, field, value):
    corun, cache, rows, x = _parts()
    setattr(cache, field, value)
    c, r, h = C.byref(cache), C.byref(rows), C.byref(x)
    assert lib.corun_kv8_append(c, r, h, h, 1, None, None, None, None, 0, None, None) == corun.EINVAL
    assert lib.corun_kv8_attend(c, r, 1, h, h, 1, 32, 0.1, 0, None, BASE, 1 << 40, None) == corun.EINVAL
    assert lib.corun_kv8_evict(c, BASE, 8, 4, BASE, BASE, BASE, BASE, 64, 4, 16, BASE, BASE, 1 << 40, None) == corun.EINVAL


@pytest.mark.parametrize("field,value", [("block_table", None), ("ctx", None), ("max_blocks", 0), ("max_blocks", 2**26), ("B", 0), ("B", 65536),
                                         ("T", -1), ("T", 5)])
def test_bad_rows_are_refused(lib, field, value):
    corun, cache, rows, x = _parts()
    setattr(rows, field, value)
    c, r, h = C.byref(cache), C.byref(rows), C.byref(x)
    assert lib.corun_kv8_append(c, r, h, h, 1, None, None, None, None, 0, None, None) == corun.EINVAL
    assert lib.corun_kv8_attend(c, r, 1, h, h, 1, 32, 0.1, 0, None, BASE, 1 << 40, None) == corun.EINVAL


def test_append_refusals(lib):
    corun, cache, rows, x = _parts()
    rope = corun.Rope(128)
    wide = corun.Rope(130)
    c, r, h = C.byref(cache), C.byref(rows), C.byref(x)
    for a in ((None, r, h, h, 1, None, None, None, None, 0), (c, None, h, h, 1, None, None, None, None, 0),
              (c, r, None, h, 1, None, None, None, None, 0), (c, r, h, None, 1, None, None, None, None, 0),
              (c, r, h, h, 3, None, None, None, None, 0), (c, r, h, h, 1, rope._h, None, None, None, 0),
              (c, r, h, h, 1, wide._h, BASE, None, None, 0), (c, r, h, h, 1, None, None, h, None, 8), (c, r, h, h, 1, None, None, h, h, 0),
              (c, r, C.byref(corun.Heads(BASE + 1, 1, 1)), h, 1, None, None, None, None, 0)):
        assert lib.corun_kv8_append(*a, None, None) == corun.EINVAL


def test_attend_refusals(lib):
    corun, cache, rows, x = _parts()
    need = lib.corun_kv8_attend_bytes(4, 4, 1, 32, 8, 128, 16, 8, 0)
    assert need > 0
    ok = dict(max_new=1, q=C.byref(x), out=C.byref(x), dtype=1, n_q=32, scale=0.1, window=0, mass=None, ws=BASE, n=need)
    for bad in (dict(max_new=0), dict(max_new=2), dict(q=None), dict(out=None), dict(dtype=0), dict(dtype=3), dict(n_q=0), dict(n_q=12),
                dict(n_q=8 * 33), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(ws=None),
                dict(ws=BASE + 16), dict(n=need - 1), dict(q=C.byref(corun.Heads(BASE + 8, 1024, 128))),
                dict(out=C.byref(corun.Heads(BASE, 1020, 128)))):
        a = dict(ok, **bad)
        assert lib.corun_kv8_attend(C.byref(cache), C.byref(rows), a["max_new"], a["q"], a["out"], a["dtype"], a["n_q"], a["scale"], a["window"],
                                    a["mass"], a["ws"], a["n"], None) == corun.EINVAL, bad
    rows.B = rows.T = 513
    assert lib.corun_kv8_attend(C.byref(cache), C.byref(rows), 1, C.byref(x), C.byref(x), 1, 32, 0.1, 0, None, BASE, 1 << 40, None) == corun.EINVAL
    rows.B, rows.T, rows.cu = 4, 40, BASE                       # 9 tokens of 4 heads: more than the weights are added up for
    assert lib.corun_kv8_attend(C.byref(cache), C.byref(rows), 9, C.byref(x), C.byref(x), 1, 32, 0.1, 0, BASE, BASE, 1 << 40, None) == corun.EINVAL
    assert lib.corun_kv8_sync(None, None) == corun.EINVAL
    for a in ((0, 1, 1, 8, 8, 64, 16, 1, 0), (1, 0, 1, 8, 8, 64, 16, 1, 0), (1, 1, 1, 8, 8, 64, 16, 0, 0)):
        assert lib.corun_kv8_attend_bytes(*a) == 0


def test_evict_refusals(lib):
    corun, cache, rows, x = _parts()
    need = lib.corun_kv8_evict_bytes(4, 8, 64)
    ok = [BASE, 8, 4, BASE, BASE, BASE, BASE, 64, 4, 16, BASE, BASE, need]
    for at, v in ((0, None), (1, 0), (1, 65537), (2, 0), (2, 65536), (3, None), (4, None), (5, None), (6, None), (7, 0), (7, 129), (8, -1), (9, -1),
                  (9, 61), (10, None), (11, None), (11, BASE + 64), (12, need - 1)):
        a = list(ok)
        a[at] = v
        assert lib.corun_kv8_evict(C.byref(cache), *a, None) == corun.EINVAL, (at, v)
    assert lib.corun_kv8_evict_bytes(0, 8, 64) == 0


def test_python_checks():
    """What the binding refuses before it calls the library."""
    from paper_2608_14376_b200 import corun

    with pytest.raises(ValueError):                             # a pool of another type
        corun.Kv8Cache(4, 2, 64, pool=torch.zeros(4, 2, 2, 16, 64), exps=torch.zeros(4, 2, 2, dtype=torch.int8))
    cache = corun.Kv8Cache(4, 2, 64, device="cpu")
    k = torch.zeros(1, 2, 64)
    ctx, table = torch.ones(1, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError):                             # no CUDA tensor
        cache.append(k, k, ctx, table)
    with pytest.raises(ValueError):
        cache.append(k, k[:, :1], ctx, table)
    with pytest.raises(ValueError):
        cache.append(k, k, ctx.long(), table)
    with pytest.raises(ValueError):
        cache.append(k.transpose(1, 2).contiguous().transpose(1, 2), k, ctx, table)
    with pytest.raises(ValueError):
        cache.append(k, k, ctx, table, rope=corun.Rope(64))
    with pytest.raises(ValueError):
        corun.Rope(64).apply(k.double(), ctx)
    att = corun.Kv8Attention(1, 4, 2, 64, 4)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        att.run(q.float(), cache, ctx, table, 0.1)
    with pytest.raises(ValueError):
        att.run(q, cache, ctx, table[:, :3].contiguous(), 0.1)
    with pytest.raises(ValueError):
        att.run(torch.zeros(2, 4, 64, dtype=torch.bfloat16), cache, ctx, table, 0.1)
    with pytest.raises(ValueError):
        cache.evict(ctx, table, None, ctx, 8)
