"""The cache operators refuse what they cannot do, before touching a device (no GPU needed)."""

import ctypes as C

import pytest

P16 = 0x1000  # (an aligned address that nothing reads)


def good(fsb):
    cache = fsb.fs_kv_cache(8, 2, 16, 128, P16, P16, P16, P16, 2 * 16 * 128, 16 * 128, 128)
    batch = fsb.fs_kv_batch(3, 5, 2, 40, 4, 0, P16, P16, P16)
    rows = fsb.fs_kv_rows(P16, 1024, 128)
    new = fsb.fs_kv_new(0, 4, 128, 0, 100, 0, rows, rows, rows, rows, P16, P16)
    query = fsb.fs_kv_query(0, 4, 0.1, 0, rows, rows)
    return cache, batch, new, query


CACHE = [("pages", 0), ("heads", 0), ("heads", 1025), ("page_tokens", 8), ("page_tokens", 48), ("page_tokens", 256),
         ("dim", 96), ("dim", 256), ("k", None), ("v", P16 + 8), ("k_scale", None), ("v_scale", P16 + 2),
         ("page_stride", 24), ("head_stride", 0), ("token_stride", 64), ("token_stride", 1 << 41)]
BATCH = [("batch", -1), ("batch", 65536), ("tokens", -1), ("max_new", 6), ("max_new", -1), ("max_length", -1),
         ("max_length", (1 << 30) + 1), ("max_length", 65), ("table_stride", -1), ("page_table", None), ("length", None),
         ("q_start", None)]


def refused(fsb, rc):
    assert rc == fsb.FS_EINVAL and fsb.fs_last_error()


@pytest.mark.parametrize("field,value", CACHE)
def test_cache(fsb, field, value):
    cache, batch, new, query = good(fsb)
    setattr(cache, field, value)
    L, n = fsb.lib(), C.c_int64()
    refused(fsb, L.fs_kv_append(C.byref(cache), C.byref(batch), C.byref(new), P16, 1 << 40, None))
    refused(fsb, L.fs_kv_attend(C.byref(cache), C.byref(batch), C.byref(query), P16, 1 << 40, None))
    refused(fsb, L.fs_kv_workspace_bytes(C.byref(cache), C.byref(batch), 4, C.byref(n)))


@pytest.mark.parametrize("field,value", BATCH)
def test_batch(fsb, field, value):
    cache, batch, new, query = good(fsb)
    setattr(batch, field, value)
    L = fsb.lib()
    refused(fsb, L.fs_kv_append(C.byref(cache), C.byref(batch), C.byref(new), P16, 1 << 40, None))
    refused(fsb, L.fs_kv_attend(C.byref(cache), C.byref(batch), C.byref(query), P16, 1 << 40, None))


@pytest.mark.parametrize("field,value", [("dtype", 2), ("q_heads", 0), ("rot", 4), ("rot", 136), ("rot", -8),
                                         ("interleaved", 2), ("angle_rows", 0), ("cos", None), ("sin", P16 + 4)])
def test_append(fsb, field, value):
    cache, batch, new, _ = good(fsb)
    setattr(new, field, value)
    refused(fsb, fsb.lib().fs_kv_append(C.byref(cache), C.byref(batch), C.byref(new), P16, 1 << 40, None))


@pytest.mark.parametrize("rows", ["k", "v", "q", "q_out"])
@pytest.mark.parametrize("field,value", [("data", None), ("data", P16 + 8), ("token_stride", 4), ("head_stride", -8)])
def test_append_rows(fsb, rows, field, value):
    cache, batch, new, _ = good(fsb)
    setattr(getattr(new, rows), field, value)
    refused(fsb, fsb.lib().fs_kv_append(C.byref(cache), C.byref(batch), C.byref(new), P16, 1 << 40, None))


@pytest.mark.parametrize("field,value", [("dtype", -1), ("q_heads", 3), ("q_heads", 0), ("scale", float("nan")),
                                         ("scale", float("inf")), ("window", -1)])
def test_attend(fsb, field, value):
    cache, batch, _, query = good(fsb)
    setattr(query, field, value)
    refused(fsb, fsb.lib().fs_kv_attend(C.byref(cache), C.byref(batch), C.byref(query), P16, 1 << 40, None))


@pytest.mark.parametrize("rows", ["q", "out"])
@pytest.mark.parametrize("field,value", [("data", None), ("data", P16 + 2), ("token_stride", 12)])
def test_attend_rows(fsb, rows, field, value):
    cache, batch, _, query = good(fsb)
    setattr(getattr(query, rows), field, value)
    refused(fsb, fsb.lib().fs_kv_attend(C.byref(cache), C.byref(batch), C.byref(query), P16, 1 << 40, None))


def test_workspace_and_null_structs(fsb):
    cache, batch, new, query = good(fsb)
    L = fsb.lib()
    for ws, n in ((None, 1 << 40), (P16 + 16, 1 << 40), (P16, 256)):
        refused(fsb, L.fs_kv_append(C.byref(cache), C.byref(batch), C.byref(new), ws, n, None))
    refused(fsb, L.fs_kv_append(None, C.byref(batch), C.byref(new), P16, 1 << 40, None))
    refused(fsb, L.fs_kv_append(C.byref(cache), None, C.byref(new), P16, 1 << 40, None))
    refused(fsb, L.fs_kv_append(C.byref(cache), C.byref(batch), None, P16, 1 << 40, None))
    refused(fsb, L.fs_kv_attend(C.byref(cache), C.byref(batch), None, P16, 1 << 40, None))
    refused(fsb, L.fs_kv_workspace_bytes(C.byref(cache), C.byref(batch), 3, C.byref(C.c_int64())))
    refused(fsb, L.fs_kv_workspace_bytes(C.byref(cache), C.byref(batch), 4, None))
    refused(fsb, L.fs_kv_check(None, None))


def test_calls_without_tokens_do_nothing(fsb):
    cache, batch, new, query = good(fsb)
    L = fsb.lib()
    for field in ("batch", "tokens"):
        _, b, _, _ = good(fsb)
        setattr(b, field, 0)
        if field == "tokens":
            b.max_new = 0
        assert L.fs_kv_append(C.byref(cache), C.byref(b), C.byref(new), P16, 1 << 40, None) == fsb.FS_OK
        assert L.fs_kv_attend(C.byref(cache), C.byref(b), C.byref(query), P16, 1 << 40, None) == fsb.FS_OK


def test_the_binding_checks_tensors(fsb):
    """Shapes, types and places that the binding sees before the library does."""
    import torch

    k = torch.zeros(4, 2, 16, 128, dtype=torch.uint8)
    s = torch.zeros(4, 2)
    with pytest.raises(ValueError, match="CUDA"):
        fsb.KvCache(k, k, s, s)
    with pytest.raises(ValueError, match="equal strides"):
        fsb.KvCache(k, k.transpose(1, 2).contiguous().transpose(1, 2), s, s)
    with pytest.raises(ValueError, match="float8"):
        fsb.KvCache(k.float(), k.float(), s, s)
    with pytest.raises(ValueError, match="float32"):
        fsb.KvCache(k, k, s.double(), s)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="page_table"):
        fsb.KvBatch(torch.zeros(2, 4, dtype=torch.int32), i, torch.zeros(4, dtype=torch.int32), 0, 0, 0)
    with pytest.raises(ValueError, match="int32"):
        fsb.KvBatch(torch.zeros(3, 4, dtype=torch.int64), i, torch.zeros(4, dtype=torch.int32), 0, 0, 0)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        fsb._kv_dtype(s)


def test_more_tokens_than_sequences_can_hold(fsb):
    cache, batch, new, query = good(fsb)
    batch.tokens = 7  # three sequences of at most two new tokens
    refused(fsb, fsb.lib().fs_kv_append(C.byref(cache), C.byref(batch), C.byref(new), P16, 1 << 40, None))
    batch.tokens, batch.max_new = 1 << 29, 1 << 29  # times four query heads
    refused(fsb, fsb.lib().fs_kv_attend(C.byref(cache), C.byref(batch), C.byref(query), P16, 1 << 40, None))
