"""Sizes at the limits of awe_cache_attend: what it refuses, awe_cache_attend_workspace_bytes refuses too, and what it accepts has a
workspace whose bytes are counted without overflow (CPU only)."""
import ctypes

import pytest

from paper_2609_24519_amd import awe

P = 1 << 40  # never dereferenced


def arguments(rows, max_rows, sequences, max_length, heads=1, dim=64):
    return (awe.CacheStruct(P, P, P, P, 10, heads, dim, 16),
            awe.BatchStruct(sequences, P, P, P, (max_length + 15) // 16, rows, max_rows, max_length))


def workspace(c, b, q_heads):
    n = ctypes.c_size_t(0)
    return awe.lib().awe_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(b), q_heads, ctypes.byref(n)), n.value


def attend_without_workspace(c, b, q_heads):
    """The status of a call that is refused (nothing else may be asked of it: the pointers are none)."""
    d = c.head_dim
    return awe.lib().awe_cache_attend(ctypes.byref(c), ctypes.byref(b), P, q_heads * d, d, q_heads, awe.BF16, 1.0, 1,
                                      P, q_heads * d, d, None, 0, None, None)


@pytest.mark.parametrize("q_heads,rows,sequences", [(65535, 1 << 27, (1 << 24) - 1), (65535, 1 << 27, 1), (64, 1 << 25, 1 << 20),
                                                    (65535, (1 << 14) + 1, 4000)])
def test_what_attention_refuses_has_no_workspace(q_heads, rows, sequences):
    c, b = arguments(rows, rows, sequences, 1 << 20)
    assert attend_without_workspace(c, b, q_heads) == awe.ERR_UNSUPPORTED
    assert workspace(c, b, q_heads) == (awe.ERR_UNSUPPORTED, 0)


@pytest.mark.parametrize("heads,dim", [(1, 64), (8, 128), (64, 256)])
@pytest.mark.parametrize("sequences", [1, 3, 60, 700])
@pytest.mark.parametrize("max_rows,share", [(1, 1), (1, 64), (3, 8), (40, 1)])
@pytest.mark.parametrize("max_length", [1, 4096, 1 << 20, 1 << 30])
def test_workspace_holds_every_part(heads, dim, sequences, max_rows, share, max_length):
    c, b = arguments(max_rows * sequences, max_rows, sequences, max_length, heads, dim)
    status, n = workspace(c, b, heads * share)
    assert status == awe.OK
    # a part per split of a column: 4 + dim floats; refused without a workspace wherever there is one
    assert n % (sequences * heads * max_rows * share * (dim + 4) * 4) == 0
    assert n == 0 or attend_without_workspace(c, b, heads * share) == awe.ERR_WORKSPACE
