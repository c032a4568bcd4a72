"""The C ABI of quantised inference on the host (CPU only): refusals before anything is enqueued, empty
calls, workspaces, and the checks of the torch conveniences."""
import ctypes

import pytest
import torch

from paper_2609_24519_amd import awe

P = 1 << 40  # never dereferenced: every call below ends in its argument checks


def w4(**kw):
    a = dict(M=4, N=8, K=64, X=P, ldx=64, x_type=awe.BF16, x_scales=None, W=P, ldw=32, w_scales=P, lds=2,
             s_type=awe.F32, zeros=None, ldz=0, group=32, Y=P, ldy=8, y_type=awe.BF16)
    a.update(kw)
    return awe.lib().awe_gemm_w4(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(M=-1), dict(N=-1), dict(K=-1), dict(x_type=awe.F32), dict(x_type=awe.I32), dict(x_type=77),
    dict(s_type=awe.I8), dict(y_type=awe.I32), dict(y_type=awe.I8), dict(x_scales=P), dict(group=0), dict(group=-32),
    dict(group=48), dict(group=63), dict(X=None), dict(W=None), dict(w_scales=None), dict(Y=None), dict(ldx=63),
    dict(ldw=31), dict(lds=1), dict(zeros=P, ldz=1), dict(ldy=7), dict(X=P + 1), dict(Y=P + 1), dict(w_scales=P + 2),
    dict(x_type=awe.I8, x_scales=P + 2), dict(K=63, ldw=31)])
def test_w4_refuses(bad):
    assert w4(**bad) == awe.ERR_INVALID_VALUE
    assert awe.lib().awe_last_error().decode() != ""


def test_w4_sizes():
    assert w4(M=0, X=None, Y=None) == awe.OK and w4(N=0, W=None, Y=None) == awe.OK
    assert w4(M=1 << 31) == awe.ERR_UNSUPPORTED and w4(N=1 << 31, ldy=1 << 31) == awe.ERR_UNSUPPORTED
    assert w4(K=1 << 31, ldx=1 << 31) == awe.ERR_UNSUPPORTED
    # rows 16 MiB apart and more, up to strides whose bytes pass 64 bits
    for far in (1 << 24, 1 << 62):
        assert w4(ldx=far // 2) == awe.ERR_UNSUPPORTED and w4(ldw=far) == awe.ERR_UNSUPPORTED
        assert w4(lds=far // 4) == awe.ERR_UNSUPPORTED and w4(zeros=P, ldz=far) == awe.ERR_UNSUPPORTED
    assert w4(ldx=1 << 62) == awe.ERR_UNSUPPORTED and w4(lds=1 << 62) == awe.ERR_UNSUPPORTED


def cache(**kw):
    a = dict(k=P, v=P, k_scales=P, v_scales=P, num_blocks=10, heads=2, head_dim=64, block=16)
    a.update(kw)
    return awe.CacheStruct(*a.values())


def batch(**kw):
    a = dict(sequences=2, starts=P, lengths=P, blocks=P, ld_blocks=4, rows=5, max_rows=3, max_length=64)
    a.update(kw)
    return awe.BatchStruct(*a.values())


def tokens(load, c=None, b=None, **kw):
    a = dict(k=P, k_row=128, k_head=64, v=P, v_row=128, v_head=64, dtype=awe.BF16, flag=None)
    a.update(kw)
    f = awe.lib().awe_cache_load if load else awe.lib().awe_cache_store
    return f(ctypes.byref(c or cache()), ctypes.byref(b or batch()), *a.values(), None)


def attend(c=None, b=None, **kw):
    a = dict(q=P, q_row=256, q_head=64, q_heads=4, dtype=awe.BF16, scale=1.0, causal=1, out=P, out_row=256,
             out_head=64, ws=None, ws_bytes=0, flag=None)
    a.update(kw)
    return awe.lib().awe_cache_attend(ctypes.byref(c or cache()), ctypes.byref(b or batch()), *a.values(), None)


CALLS = [lambda **k: tokens(False, **k), lambda **k: tokens(True, **k), attend]


@pytest.mark.parametrize("call", CALLS)
def test_cache_and_batch_refusals(call):
    for bad in (dict(num_blocks=-1), dict(heads=0), dict(k=None), dict(v=None), dict(k_scales=None),
                dict(v_scales=None), dict(k=P + 8), dict(v=P + 1), dict(k_scales=P + 2)):
        assert call(c=cache(**bad)) == awe.ERR_INVALID_VALUE, bad
    for bad in (dict(block=8), dict(block=48), dict(block=256), dict(head_dim=96), dict(head_dim=512),
                dict(head_dim=0), dict(num_blocks=1 << 31)):
        assert call(c=cache(**bad)) == awe.ERR_UNSUPPORTED, bad
    for bad in (dict(sequences=-1), dict(rows=-1), dict(max_rows=-1), dict(max_length=-1), dict(ld_blocks=-1),
                dict(ld_blocks=3), dict(starts=None), dict(lengths=None), dict(blocks=None), dict(starts=P + 2),
                dict(lengths=P + 1), dict(blocks=P + 2)):
        assert call(b=batch(**bad)) == awe.ERR_INVALID_VALUE, bad
    for bad in (dict(rows=1 << 28), dict(max_rows=1 << 28), dict(max_length=(1 << 30) + 1, ld_blocks=1 << 31),
                dict(sequences=1 << 24)):
        assert call(b=batch(**bad)) == awe.ERR_UNSUPPORTED, bad
    for nothing in (dict(sequences=0), dict(rows=0), dict(max_rows=0)):
        assert call(b=batch(**nothing, starts=None, lengths=None, blocks=None)) == awe.OK
    assert call(flag=P + 2) == awe.ERR_INVALID_VALUE
    f = awe.lib().awe_cache_store
    assert f(None, ctypes.byref(batch()), P, 1, 1, P, 1, 1, awe.BF16, None, None) == awe.ERR_INVALID_VALUE
    assert f(ctypes.byref(cache()), None, P, 1, 1, P, 1, 1, awe.BF16, None, None) == awe.ERR_INVALID_VALUE


@pytest.mark.parametrize("load", [False, True])
def test_row_refusals(load):
    for bad in (dict(k=None), dict(v=None), dict(k=P + 1), dict(v=P + 1), dict(k_row=-1), dict(v_head=-1),
                dict(dtype=awe.I8), dict(dtype=awe.I64), dict(dtype=awe.F32, k=P + 2)):
        assert tokens(load, **bad) == awe.ERR_INVALID_VALUE, bad
    assert tokens(load, k_row=1 << 41) == awe.ERR_UNSUPPORTED
    if load:  # written elements that share memory
        for bad in (dict(k_row=0), dict(k_row=127), dict(v_head=63), dict(v_row=64, v_head=64)):
            assert tokens(load, **bad) == awe.ERR_INVALID_VALUE, bad
        # rows * stride past 64 bits
        far = dict(k_row=1 << 40, k_head=1 << 39)
        assert tokens(load, b=batch(rows=(1 << 23) + 1, max_rows=1), c=cache(heads=3), **far) == awe.ERR_INVALID_VALUE


def test_attend_refusals():
    for bad in (dict(q=None), dict(out=None), dict(q=P + 1), dict(out=P + 1), dict(q_heads=3), dict(q_heads=0),
                dict(q_heads=-4), dict(dtype=awe.F32), dict(dtype=awe.I8), dict(q_row=-1), dict(out_row=255),
                dict(out_head=63), dict(out_row=0)):
        assert attend(**bad) == awe.ERR_INVALID_VALUE, bad
    assert attend(q_heads=65536) == awe.ERR_UNSUPPORTED


def test_attend_workspace():
    L, n = awe.lib(), ctypes.c_size_t(7)
    c, b = cache(), batch()
    assert L.awe_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 4, None) == awe.ERR_INVALID_VALUE
    assert L.awe_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 3,
                                              ctypes.byref(n)) == awe.ERR_INVALID_VALUE
    assert awe.cache_attend_workspace_bytes(c, batch(sequences=0), 4) == 0
    assert awe.cache_attend_workspace_bytes(c, batch(rows=0), 4) == 0


def test_conveniences_check_shapes():
    x, w, s = torch.zeros(3, 64), torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(5, 2)
    h = x.to(torch.bfloat16)
    for args, kw in (((x, w, s, 32), {}), ((h, w[:, :31], s, 32), {}), ((h, w.to(torch.int8), s, 32), {}),
                     ((h, w, s[:, :1], 32), {}), ((h, w, s, 0), {}), ((h, w, s, 32), dict(zeros=torch.zeros(5, 2))),
                     ((h, w, s, 32), dict(zeros=torch.zeros(5, 1, dtype=torch.uint8))), ((h[0], w, s, 32), {}),
                     ((x.to(torch.int8), w, s, 32), dict(x_scales=torch.zeros(2))),
                     ((h, w, s, 32), dict(out_dtype=torch.int32))):
        with pytest.raises(ValueError):
            awe.matmul_w4(*args, **kw)
    i8 = lambda *n: torch.zeros(*n, dtype=torch.int8)  # noqa: E731
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    f = torch.zeros(4, 2)
    c = awe.Cache(i8(4, 2, 16, 64), i8(4, 2, 64, 16), f, f)
    for bad in ((i8(4, 2, 16, 64), i8(4, 2, 16, 64), f, f), (i8(4, 2, 16, 64), i8(4, 2, 64, 16), f, torch.zeros(4)),
                (torch.zeros(4, 2, 16, 64), i8(4, 2, 64, 16), f, f),
                (i8(4, 2, 64, 16).transpose(2, 3), i8(4, 2, 64, 16), f, f)):
        with pytest.raises(ValueError):
            awe.Cache(*bad)
    awe.Batch(i32(3), i32(2), i32(2, 4), 5, 3, 64)
    for bad in ((i32(2), i32(2), i32(2, 4)), (i32(3), i32(2), i32(3, 4)), (i32(3).long(), i32(2), i32(2, 4)),
                (i32(6)[::2], i32(2), i32(2, 4)), (i32(3), i32(2), i32(1, 4).expand(2, 4))):
        with pytest.raises(ValueError):
            awe.Batch(*bad, 5, 3, 64)
    b = awe.Batch(i32(3), i32(2), i32(2, 4), 5, 3, 64)
    q = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        awe.store_tokens(c, b, q, q[:, :1])
    with pytest.raises(ValueError):
        awe.store_tokens(c, b, q, q.half())
    with pytest.raises(ValueError):
        awe.attend(c, b, q[:4], 1.0)
    with pytest.raises(ValueError):
        awe.attend(c, b, q.float(), 1.0)
    for flag in (torch.zeros(1), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(ValueError):
            awe.attend(c, b, q, 1.0, d_range_flag=flag)
    far = [torch.zeros(s, dtype=t, device="meta") for s, t in (((4, 2), torch.float32), ((2,), torch.int32))]
    with pytest.raises(ValueError):  # tensors of two devices
        awe.Cache(i8(4, 2, 16, 64), i8(4, 2, 64, 16), f, far[0])
    with pytest.raises(ValueError):
        awe.Batch(i32(3), far[1], i32(2, 4), 5, 3, 64)
    for call in (lambda: awe.matmul_w4(h, w, s, 32), lambda: awe.store_tokens(c, b, q, q),
                 lambda: awe.attend(c, b, q, 1.0)):  # tensors of the host
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):  # past the entries of the table
        awe.attend(c, awe.Batch(i32(3), i32(2), i32(2, 3), 5, 3, 64), q, 1.0)
