"""Calls of the 8-bit cache's operators that come back before any CUDA call: calls without tokens, objects that were closed, workspaces."""
import ctypes as C

import pytest
import torch

from tests.test_kv8_oracle import BASE, _parts, lib  # noqa: F401 (lib: a fixture)


def test_no_tokens_need_no_data(lib):
    """A call without tokens reads no tensor: an empty one has no address."""
    corun, cache, rows, x = _parts()
    rows.T, rows.cu = 0, BASE
    c, r, none = C.byref(cache), C.byref(rows), C.byref(corun.Heads(None, 1024, 128))
    rope = corun.Rope(128)
    assert lib.corun_kv8_append(c, r, none, none, 1, None, None, None, None, 0, None, None) == corun.OK
    assert lib.corun_kv8_append(c, r, none, none, 1, rope._h, None, none, none, 32, None, None) == corun.OK
    assert lib.corun_kv8_attend(c, r, 4, none, none, 1, 32, 0.1, 0, None, None, 0, None) == corun.OK
    # the rest is checked all the same
    assert lib.corun_kv8_append(c, r, none, none, 3, None, None, None, None, 0, None, None) == corun.EINVAL
    assert lib.corun_kv8_append(c, r, none, none, 1, None, None, none, none, 0, None, None) == corun.EINVAL
    assert lib.corun_kv8_append(c, r, None, none, 1, None, None, None, None, 0, None, None) == corun.EINVAL
    assert lib.corun_kv8_attend(c, r, 0, none, none, 1, 32, 0.1, 0, None, None, 0, None) == corun.EINVAL
    assert lib.corun_kv8_attend(c, r, 4, none, none, 1, 12, 0.1, 0, None, None, 0, None) == corun.EINVAL
    assert lib.corun_kv8_attend(c, r, 4, none, None, 1, 32, 0.1, 0, None, None, 0, None) == corun.EINVAL
    rows.cu = None                                              # one token each: not none
    assert lib.corun_kv8_append(c, r, none, none, 1, None, None, None, None, 0, None, None) == corun.EINVAL


def test_a_closed_rope_is_refused(lib):
    """append with a closed ``Rope`` does not go on without rotating."""
    from paper_2608_14376_b200 import corun

    rope = corun.Rope(64)
    rope.close()
    rope.close()
    cache = corun.Kv8Cache(4, 2, 64, device="cpu")
    k, one = torch.zeros(1, 2, 64), torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="closed"):
        cache.append(k, k, one, torch.zeros(1, 4, dtype=torch.int32), positions=one, rope=rope)
    with pytest.raises(ValueError, match="closed"):
        rope.apply(k, one)


@pytest.mark.parametrize("sinks,recent", [(2 ** 32, 4), (4, 2 ** 32), (2 ** 32 + 4, 2 ** 32 + 4), (4, -2 ** 32 + 4)])
def test_evict_refuses_counts_beyond_32_bits(sinks, recent):
    """What the library would get in 32 bits is another number."""
    from paper_2608_14376_b200 import corun

    cache = corun.Kv8Cache(4, 2, 64, device="cpu")
    one, table = torch.ones(1, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError, match="sinks"):
        cache.evict(one, table, torch.zeros(1, 2, 64), one, 32, sinks=sinks, recent=recent)


def test_workspace_goes_by_the_tokens_that_there_are(lib):
    """A call's partial results: a column per token and query head, where rows times the most columns of a row would be more."""
    need = lambda B, T, max_new: lib.corun_kv8_attend_bytes(B, T, max_new, 32, 8, 128, 16, 2048, 0)
    splits = 128                                                # tables of 32768 tokens: 256 tiles of 128
    part = lambda columns: 8 * splits * columns * (128 + 2) * 4  # a column's running output, frame and sum
    for B, T, max_new, columns in ((512, 512, 1, 512 * 4), (512, 512 + 511, 512, 1023 * 4), (64, 64 + 63, 64, 127 * 4), (64, 4096, 4096, 64 * 32),
                                   (3, 9, 5, 9 * 4), (1, 300, 300, 32)):
        assert part(columns) <= need(B, T, max_new) <= part(columns) + 4096, (B, T, max_new)
