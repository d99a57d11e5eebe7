"""What the multi-token operators refuse, before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2609_37988_amd import kvk

P0 = 1 << 20  # an aligned address that is no GPU memory
I32 = ctypes.c_int32


def _arr(vals):
    return None if vals is None else (I32 * len(vals))(*vals)


def _strides(*triples):
    return (ctypes.c_int64 * (3 * len(triples)))(*[x for t in triples for x in t])  # kvk_strides entries


def _refused(status, want, *words):
    assert status == want, (status, kvk.last_error())
    for w in words:
        assert w in kvk.last_error(), kvk.last_error()


def _prompt(hq=4, hkv=2, d=64, lens=(5, 3), q=P0, k=P0, v=P0, strides=None, scale=0.1, out=P0, lse=None, n=None):
    return kvk.load().kvk_prompt_attention(hq, hkv, d, len(lens) if n is None else n, _arr(lens), q, k, v, strides, scale,
                                           out, lse, None)


def _weight(hq=4, hkv=2, d=64, lens=(5, 3), q=P0, k=P0, strides=None, lse=P0, scale=0.1, weight=P0, ws=P0, ws_bytes=1 << 20):
    return kvk.load().kvk_attention_weight(hq, hkv, d, len(lens), _arr(lens), q, k, strides, lse, scale, weight, ws,
                                           ws_bytes, None)


@pytest.mark.parametrize("call", [_prompt, _weight])
def test_prompt_sizes(call):
    _refused(call(hq=5), kvk.ERR_INVALID, "5 query heads over 2")
    _refused(call(hkv=0), kvk.ERR_INVALID)
    _refused(call(hq=0), kvk.ERR_INVALID)
    _refused(call(d=96), kvk.ERR_UNSUPPORTED, "head_dim 96")
    _refused(call(lens=()), kvk.ERR_INVALID, "no sequences")
    _refused(call(lens=(4, -1)), kvk.ERR_INVALID, "sequence 1")
    _refused(call(lens=[1] * 257), kvk.ERR_UNSUPPORTED, "257 sequences")
    _refused(call(lens=(2**31 - 1, 2**31 - 1)), kvk.ERR_UNSUPPORTED, "tokens in all")
    _refused(call(scale=float("nan")), kvk.ERR_INVALID, "finite")
    _refused(call(scale=float("inf")), kvk.ERR_INVALID, "finite")
    assert call(lens=(0, 0)) == kvk.OK  # nothing to do
    _refused(call(), kvk.ERR_INVALID, "not GPU-accessible")


def test_prompt_buffers_and_strides():
    for name in ("q", "k", "v", "out"):
        _refused(_prompt(**{name: None}), kvk.ERR_INVALID, "NULL")
        _refused(_prompt(**{name: P0 + 8}), kvk.ERR_INVALID, "misaligned")
    _refused(_prompt(lse=P0 + 2), kvk.ERR_INVALID, "misaligned")
    ok = (0, 64, 256)
    _refused(_prompt(strides=_strides((0, 64, 260), ok, ok, ok)), kvk.ERR_INVALID, "q strides")
    _refused(_prompt(strides=_strides(ok, (0, 60, 256), ok, ok)), kvk.ERR_INVALID, "k strides")
    _refused(_prompt(strides=_strides(ok, ok, (4, 64, 256), ok)), kvk.ERR_INVALID, "v strides")
    _refused(_prompt(strides=_strides(ok, ok, (0, -64, 256), ok)), kvk.ERR_INVALID, "v strides")
    _refused(_prompt(strides=_strides(ok, ok, ok, (0, 0, 256))), kvk.ERR_INVALID, "overlap")
    _refused(_prompt(strides=_strides(ok, ok, ok, (0, 64, 32))), kvk.ERR_INVALID, "overlap")
    _refused(_prompt(strides=_strides((0, 0, 0), ok, ok, ok)), kvk.ERR_INVALID, "not GPU-accessible")  # inputs may repeat


def test_prompt_rows_written_do_not_overlap():
    """out strides of 4 heads of 64 and sequences of 5 and 3 tokens, or one head."""
    ok = (0, 64, 256)

    def out(*s, **kw):
        return _prompt(strides=_strides(ok, ok, ok, s), **kw)

    for bad in ((0, 64, 64), (0, 64, 192), (0, 504, 64), (64, 64, 512), (504, 64, 256), (1272, 320, 64), (256, 64, 256)):
        _refused(out(*bad), kvk.ERR_INVALID, "out rows overlap")
    # token-major, head-major, sequence-major, head above sequence, token above both
    for fine in ((0, 64, 256), (0, 512, 64), (1280, 64, 256), (1280, 320, 64), (320, 640, 64), (64, 128, 512)):
        _refused(out(*fine), kvk.ERR_INVALID, "not GPU-accessible")
    _refused(out(0, 0, 64, hq=2, hkv=2), kvk.ERR_INVALID, "out rows overlap")
    _refused(out(0, 0, 64, hq=1, hkv=1), kvk.ERR_INVALID, "not GPU-accessible")          # one head: its stride is not taken
    _refused(out(0, 64, 0, lens=(1,)), kvk.ERR_INVALID, "not GPU-accessible")            # one token
    _refused(out(0, 64, 0, lens=(1, 1)), kvk.ERR_INVALID, "out rows overlap")
    _refused(out(2**62, 2**61, 64), kvk.ERR_INVALID, "out rows overlap")


def test_weight_buffers():
    for name in ("q", "k", "lse", "weight", "ws"):
        _refused(_weight(**{name: None}), kvk.ERR_INVALID, "NULL")
    for name, off in (("q", 8), ("k", 8), ("lse", 2), ("weight", 2), ("ws", 128)):
        _refused(_weight(**{name: P0 + off}), kvk.ERR_INVALID, "misaligned")
    _refused(_weight(ws_bytes=4 * 4 * 8 - 1), kvk.ERR_BUFFER, "workspace")
    _refused(_weight(strides=_strides((0, 64, 260), (0, 64, 128))), kvk.ERR_INVALID, "q strides")
    assert kvk.attention_weight_workspace_bytes(4, 2, 64, [5, 3]) >= 4 * 4 * 8
    assert kvk.attention_weight_workspace_bytes(4, 4, 64, [5, 3]) == 0
    _refused(_weight(hkv=4, ws=None, ws_bytes=0), kvk.ERR_INVALID, "not GPU-accessible")  # one head per KV head


def _table(kind=kvk.GQA, **kw):
    a = dict(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, batch=3, max_tokens=100)
    if kind == kvk.MLA:
        a.update(n_q_heads=8, head_dim=128, latent_dim=256, rope_dim=64, nope_dim=128, v_dim=128)
    a.update(kw)
    plan = [(0, 8, 256 if kind == kvk.MLA else 0), (1, 8)]
    return kvk.layer_table(kvk.make_dims(kind, **a), kvk.make_plan(plan))


def test_keep_heaviest():
    lib = kvk.load()

    def call(t, weight=P0, n=50, recent=0, out=P0, ws=None, ws_bytes=0):
        return lib.kvk_keep_heaviest(t.handle if t else None, weight, n, recent, out, ws, ws_bytes, None)

    t = _table(keep_tokens=40)
    _refused(call(None), kvk.ERR_INVALID, "NULL table")
    _refused(call(_table()), kvk.ERR_INVALID, "does not evict")
    _refused(call(t, n=39), kvk.ERR_INVALID, "n_tokens 39")
    _refused(call(t, n=101), kvk.ERR_INVALID, "n_tokens 101")
    _refused(call(t, recent=41), kvk.ERR_INVALID, "n_recent 41")
    _refused(call(t, recent=-1), kvk.ERR_INVALID, "n_recent -1")
    _refused(call(t, weight=None), kvk.ERR_INVALID, "NULL")
    _refused(call(t, out=None), kvk.ERR_INVALID, "NULL")
    _refused(call(t, weight=P0 + 2), kvk.ERR_INVALID, "misaligned")
    _refused(call(t), kvk.ERR_INVALID, "not GPU-accessible")
    assert kvk.keep_workspace_bytes(t, 100) == 0
    t = _table(keep_tokens=40, max_tokens=40000)
    sizes = [kvk.keep_workspace_bytes(t, n) for n in (16384, 16385, 32768, 40000)]
    assert sizes[0] == 0 and sizes == sorted(sizes) and sizes[1] > 0
    _refused(call(t, n=40000), kvk.ERR_INVALID, "NULL")
    _refused(call(t, n=40000, ws=P0 + 128, ws_bytes=1 << 30), kvk.ERR_INVALID, "misaligned")
    _refused(call(t, n=40000, ws=P0, ws_bytes=sizes[-1] - 1), kvk.ERR_BUFFER, "workspace")
    _refused(call(t, n=40000, ws=P0, ws_bytes=sizes[-1]), kvk.ERR_INVALID, "not GPU-accessible")
    out = ctypes.c_size_t()
    _refused(lib.kvk_keep_workspace_bytes(_table().handle, 50, ctypes.byref(out)), kvk.ERR_INVALID, "does not evict")
    _refused(lib.kvk_keep_workspace_bytes(t.handle, 50, None), kvk.ERR_INVALID)


def _append(t, l0=0, l1=2, k=P0, v=P0, dtype=kvk.BF16, m=4, stored=(0, 10, 96), new=None, arena=P0):
    return kvk.load().kvk_append_chunk(t.handle if t else None, l0, l1, k, v, dtype, m, _arr(stored), _arr(new), arena, None)


def test_append_chunk():
    t = _table()
    _refused(_append(None), kvk.ERR_INVALID, "NULL table")
    _refused(_append(_table(kvk.MLA)), kvk.ERR_UNSUPPORTED, "kvk_append_token")
    for l0, l1 in ((-1, 1), (0, 3), (1, 1)):
        _refused(_append(t, l0, l1), kvk.ERR_INVALID, "layer range")
    for name in ("k", "v", "stored", "arena"):
        _refused(_append(t, **{name: None}), kvk.ERR_INVALID, "NULL")
    _refused(_append(t, dtype=5), kvk.ERR_INVALID, "in_dtype")
    for m in (0, -1, 101):
        _refused(_append(t, m=m), kvk.ERR_INVALID, "n_chunk")
    _refused(_append(t, stored=(0, -1, 0)), kvk.ERR_INVALID, "n_stored[1]")
    _refused(_append(t, stored=(0, 0, 101)), kvk.ERR_INVALID, "n_stored[2]")
    _refused(_append(t, stored=(0, 0, 97)), kvk.ERR_INVALID, "n_new[2] = 4")
    _refused(_append(t, new=(0, 5, 0)), kvk.ERR_INVALID, "n_new[1] = 5")
    _refused(_append(t, new=(-1, 0, 0)), kvk.ERR_INVALID, "n_new[0]")
    for name in ("k", "v", "arena"):
        _refused(_append(t, **{name: P0 + 8}), kvk.ERR_INVALID, "misaligned")
    assert _append(t, new=(0, 0, 0)) == kvk.OK          # no new tokens
    assert _append(t, 1, 2) == kvk.OK                   # only an inheriting layer
    _refused(_append(t), kvk.ERR_INVALID, "not GPU-accessible")
    big = _table(batch=300)
    _refused(_append(big, stored=[0] * 299 + [1]), kvk.ERR_UNSUPPORTED, "300 sequences of different lengths")
    _refused(_append(big, stored=[0] * 300), kvk.ERR_INVALID, "not GPU-accessible")


def _chunk(t, l0=0, l1=2, q=P0, m=4, stored=(10, 20, 100), new=None, scale=0.1, arena=P0, out=P0, ws=P0, ws_bytes=1 << 30):
    return kvk.load().kvk_chunk_attention(t.handle if t else None, l0, l1, q, m, _arr(stored), _arr(new), scale, arena, out,
                                          ws, ws_bytes, None)


def test_chunk_attention():
    t = _table()
    _refused(_chunk(None), kvk.ERR_INVALID, "NULL table")
    _refused(_chunk(_table(kvk.MLA)), kvk.ERR_UNSUPPORTED, "GQA tables")
    for l0, l1 in ((-1, 1), (0, 3), (1, 1)):
        _refused(_chunk(t, l0, l1), kvk.ERR_INVALID, "layer range")
    for name in ("q", "stored", "arena", "out", "ws"):
        _refused(_chunk(t, **{name: None}), kvk.ERR_INVALID, "NULL")
    for m in (0, 101):
        _refused(_chunk(t, m=m), kvk.ERR_INVALID, "n_chunk")
    _refused(_chunk(t, stored=(10, 101, 10)), kvk.ERR_INVALID, "n_stored[1]")
    _refused(_chunk(t, stored=(10, 3, 10)), kvk.ERR_INVALID, "n_new[1] = 4")  # more rows than tokens
    _refused(_chunk(t, new=(4, 5, 4)), kvk.ERR_INVALID, "n_new[1] = 5")
    _refused(_chunk(t, new=(4, -1, 4)), kvk.ERR_INVALID, "n_new[1] = -1")
    _refused(_chunk(t, scale=float("nan")), kvk.ERR_INVALID, "finite")
    for name, off in (("q", 8), ("arena", 8), ("out", 8), ("ws", 128)):
        _refused(_chunk(t, **{name: P0 + off}), kvk.ERR_INVALID, "misaligned")
    assert _chunk(t, new=(0, 0, 0)) == kvk.OK
    _refused(_chunk(t), kvk.ERR_INVALID, "not GPU-accessible")


def test_chunk_workspace():
    t = _table(max_tokens=50000)
    sizes = [kvk.chunk_workspace_bytes(t, 0, 2, m) for m in (1, 2, 8, 40, 1000, 50000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert kvk.chunk_workspace_bytes(t, 0, 1, 8) <= sizes[2]
    out = ctypes.c_size_t()
    call = kvk.load().kvk_chunk_workspace_bytes
    _refused(call(t.handle, 0, 2, 0, ctypes.byref(out)), kvk.ERR_INVALID)
    _refused(call(t.handle, 0, 2, 50001, ctypes.byref(out)), kvk.ERR_INVALID)
    _refused(call(t.handle, 0, 2, 1, None), kvk.ERR_INVALID)
    _refused(call(_table(kvk.MLA).handle, 0, 1, 1, ctypes.byref(out)), kvk.ERR_UNSUPPORTED)


def test_binding_refuses_a_broadcast_batch():
    """A padded batch whose sequences share one place (stride 0) has no packed meaning."""
    q, k = torch.zeros(2, 4, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    kv, lse = torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(64)
    shared = k.expand(2, 2, 8, 64)
    for args in ((q, shared, kv, q), (q, kv, shared, q), (q, kv, kv, q[:1].expand(2, 4, 8, 64)), (q[:1].expand(2, 4, 8, 64), kv, kv, q)):
        with pytest.raises(ValueError, match="broadcast"):
            kvk.prompt_attention(*args[:3], [8, 8], 0.1, args[3])
    with pytest.raises(ValueError, match="broadcast"):
        kvk.attention_weight(q, shared, lse, [8, 8], 0.1, torch.zeros(32))


def test_binding_refuses():
    """Tensors of the wrong type, layout or size, and tensors on the host."""
    x = torch.zeros(8, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    bad = [(x.float(), kv, kv, [8], x), (x, kv, kv[:, :1], [8], x), (x, kv, kv, [7], x), (x, kv, kv, [9], x), (x, kv, kv, [9, -1], x),
           (x, kv[None], kv, [8], x), (x, kv, kv, [8], x[:, :2]), (x.transpose(1, 2), kv, kv, [8], x), (x, kv, kv, [8], x)]
    for q, k, v, lens, out in bad:
        with pytest.raises(ValueError):
            kvk.prompt_attention(q, k, v, lens, 0.1, out)
    t = _table(keep_tokens=40)
    with pytest.raises(ValueError):
        kvk.keep_heaviest(t, torch.zeros(3, 2, 50), 50, 0, torch.zeros(3, 2, 40, dtype=torch.int32))
    t = _table()
    arena = torch.zeros(kvk.table_query(t).arena_bytes, dtype=torch.uint8)
    k = torch.zeros(2, 3, 2, 4, 64)
    with pytest.raises(ValueError):
        kvk.append_chunk(t, 0, 2, k, k, 0, None, arena)
    with pytest.raises(ValueError):
        kvk.append_chunk(t, 0, 1, k, k, 0, None, arena)
    with pytest.raises(ValueError):
        kvk._lengths([1, 2], 3, "n_stored")
    q = torch.zeros(2, 3, 4, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kvk.chunk_attention(t, 0, 2, q, 4, None, 0.1, arena, q, arena)
