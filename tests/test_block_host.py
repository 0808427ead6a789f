"""The operators around a block's projections refuse bad arguments on the host, before any device call (no GPU)."""
import ctypes

import pytest
import torch

INVALID, UNSUPPORTED = 1, 2
FAKE = 0x100000   # never dereferenced


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def test_norm_refusals(gs):
    f = gs.lib.gs_add_rms_norm
    far = [FAKE + (i << 20) for i in range(8)]
    x, r, w, h, y, y8, sc = far[:7]
    assert f(x, r, w, 0, 64, 1e-5, h, y, None, None, 0, None) == 0               # no rows: nothing to do
    assert f(x, r, w, -1, 64, 1e-5, h, y, None, None, 0, None) == INVALID
    assert f(x, r, w, 4, 0, 1e-5, h, y, None, None, 0, None) == INVALID
    assert f(x, r, w, 4, 64, -1.0, h, y, None, None, 0, None) == INVALID
    assert f(x, r, w, 4, 64, float("nan"), h, y, None, None, 0, None) == INVALID
    assert f(x, r, w, 4, 64, float("inf"), h, y, None, None, 0, None) == INVALID
    assert f(None, r, w, 4, 64, 1e-5, h, y, None, None, 0, None) == INVALID
    assert f(x, r, None, 4, 64, 1e-5, h, y, None, None, 0, None) == INVALID
    assert f(x, r, w, 4, 64, 1e-5, h, None, None, None, 0, None) == INVALID       # no output
    assert f(x, r, w, 4, 64, 1e-5, h, None, y8, None, 0, None) == INVALID         # 8 bits without scales
    assert f(x, r, w, 4, 64, 1e-5, h, None, y8, sc, 64, None) == UNSUPPORTED      # group
    assert f(x + 2, r, w, 4, 64, 1e-5, h, y, None, None, 0, None) == INVALID      # alignment
    assert f(x, r, w, 4, 64, 1e-5, h, h, None, None, 0, None) == INVALID          # outputs overlap
    assert f(x, r, w, 4, 64, 1e-5, h, r, None, None, 0, None) == INVALID          # y over the residual
    assert f(x, r, w, 4, 64, 1e-5, x + 16, y, None, None, 0, None) == INVALID     # h half over x
    assert f(x, r, w, 4, 64, 1e-5, h, None, x, sc, 0, None) == INVALID            # 8 bits over x


def _layer(gs, **kw):
    d = dict(x=FAKE, base=FAKE + (1 << 20), out_ptr=FAKE + (2 << 20), A=FAKE + (3 << 20), B=FAKE + (4 << 20),
             scale=FAKE + (5 << 20), inp=64, out=48, n_adapters=2, rank=8)
    d.update(kw)
    return gs._AdapterLayer(**d)


def test_adapter_refusals(gs):
    off, ids = FAKE + (6 << 20), FAKE + (7 << 20)

    def f(n, layers, n_seqs=2, T=4, o=off, i=ids):
        arr = (gs._AdapterLayer * max(1, len(layers)))(*layers)
        return gs.lib.gs_adapters_batched(n, arr, o, i, n_seqs, T, None)
    assert f(0, []) == 0 and f(1, [_layer(gs)], T=0) == 0 and f(1, [_layer(gs)], n_seqs=0) == 0
    assert f(-1, []) == INVALID and f(9, [_layer(gs)] * 9) == INVALID
    assert gs.lib.gs_adapters_batched(1, None, off, ids, 2, 4, None) == INVALID
    for bad in (dict(inp=60), dict(inp=0), dict(out=0), dict(n_adapters=0), dict(rank=0), dict(rank=-8), dict(x=None),
                dict(base=None), dict(out_ptr=None), dict(A=None), dict(B=None), dict(scale=None), dict(x=FAKE + 2),
                dict(A=FAKE + (3 << 20) + 8), dict(out_ptr=FAKE), dict(out_ptr=FAKE + (1 << 20) + 16)):
        assert f(1, [_layer(gs, **bad)]) == INVALID, bad
    assert f(1, [_layer(gs, rank=12)]) == UNSUPPORTED and f(1, [_layer(gs, rank=136)]) == UNSUPPORTED
    assert f(1, [_layer(gs, inp=1 << 30, rank=16)]) == UNSUPPORTED
    assert f(2, [_layer(gs), _layer(gs)]) == INVALID                              # one output twice
    assert f(1, [_layer(gs)], T=-1) == INVALID and f(1, [_layer(gs)], n_seqs=-1) == INVALID
    assert f(1, [_layer(gs)], o=None) == INVALID and f(1, [_layer(gs)], i=ids + 2) == INVALID


def _cache(gs, **kw):
    d = dict(k=FAKE, v=FAKE + (1 << 28), pages=4, page_size=16, kv_heads=2, head_dim=64)
    d.update(kw)
    return gs._CacheStruct(**d)


def _batch(gs, **kw):
    d = dict(offsets=FAKE + (2 << 28), kv_lens=FAKE + (3 << 28), table=FAKE + (4 << 28), n=2, table_width=3, tokens=2, max_new=1)
    d.update(kw)
    return gs._BatchStruct(**d)


BAD_CACHES = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=FAKE + 8), INVALID), (dict(pages=0), INVALID),
              (dict(kv_heads=0), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
              (dict(page_size=512), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(pages=1 << 30), UNSUPPORTED)]
BAD_BATCHES = [dict(offsets=None), dict(kv_lens=None), dict(table=None), dict(n=-1), dict(tokens=-1), dict(tokens=1 << 31),
               dict(table_width=0), dict(table_width=1 << 28), dict(max_new=-1), dict(offsets=FAKE + 2), dict(n=0)]


def test_append_refusals(gs):
    q, k, v, c, s, o = (FAKE + (i << 28) for i in range(5, 11))

    def f(cache, batch, q=q, qs=256, heads=4, k=k, ks=128, v=v, vs=128, c=c, s=s, n_pos=64, o=o):
        return gs.lib.gs_cache_append(ctypes.byref(cache), ctypes.byref(batch), q, qs, heads, k, ks, v, vs, c, s, n_pos, o, None)
    ok = _cache(gs), _batch(gs)
    assert f(ok[0], _batch(gs, tokens=0)) == 0
    assert gs.lib.gs_cache_append(None, ctypes.byref(ok[1]), q, 256, 4, k, 128, v, 128, c, s, 64, o, None) == INVALID
    for bad, st in BAD_CACHES:
        assert f(_cache(gs, **bad), ok[1]) == st, bad
    for bad in BAD_BATCHES:
        assert f(ok[0], _batch(gs, **bad)) == INVALID, bad
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(c=None), dict(s=None), dict(o=None), dict(qs=248), dict(qs=260),
                dict(ks=120), dict(vs=132), dict(heads=0), dict(n_pos=0), dict(q=q + 8), dict(o=o + 2), dict(o=q + 64), dict(o=k),
                dict(k=FAKE), dict(o=FAKE + 64), dict(c=c + 4), dict(q=q, o=q, qs=264)):
        assert f(*ok, **bad) == INVALID, bad


def test_attention_refusals(gs):
    q, o, w = (FAKE + (i << 28) for i in range(5, 8))

    def f(cache, batch, q=q, qs=256, heads=4, scale=0.1, o=o, w=w, wb=1 << 40):
        return gs.lib.gs_paged_attention(ctypes.byref(cache), ctypes.byref(batch), q, qs, heads, scale, o, w, wb, None)
    ok = _cache(gs), _batch(gs)
    assert f(ok[0], _batch(gs, tokens=0)) == 0
    for bad, st in BAD_CACHES:
        assert f(_cache(gs, **bad), ok[1]) == st, bad
    for bad in BAD_BATCHES:
        assert f(ok[0], _batch(gs, **bad)) == INVALID, bad
    for bad in (dict(q=None), dict(o=None), dict(qs=248), dict(qs=260), dict(heads=0), dict(heads=3), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(q=q + 8), dict(o=o + 2), dict(o=q), dict(o=FAKE)):
        assert f(*ok, **bad) == INVALID, bad
    assert f(*ok, heads=130, qs=130 * 64) == UNSUPPORTED                          # 65 query heads a key head
    n = ctypes.c_size_t()
    assert gs.lib.gs_paged_attention_workspace(ctypes.byref(ok[0]), ctypes.byref(ok[1]), 4, ctypes.byref(n)) == 0
    assert gs.lib.gs_paged_attention_workspace(ctypes.byref(ok[0]), ctypes.byref(ok[1]), 3, ctypes.byref(n)) == INVALID
    assert gs.lib.gs_paged_attention_workspace(ctypes.byref(ok[0]), ctypes.byref(ok[1]), 4, None) == INVALID
    if n.value:
        assert f(*ok, wb=n.value - 1) == INVALID and f(*ok, w=None) == INVALID and f(*ok, w=w + 8) == INVALID
        assert f(*ok, w=o) == INVALID


def test_binding_refuses_host_and_misshapen_tensors(gs):
    bf, x = torch.bfloat16, torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        gs.add_rms_norm(x, torch.ones(64, dtype=bf), y=x)
    with pytest.raises(ValueError, match="CUDA"):
        gs.Adapters(torch.zeros((1, 8, 64), dtype=bf), torch.zeros((1, 4, 8), dtype=bf), torch.ones(1))
    with pytest.raises(ValueError, match="CUDA"):
        gs.PagedCache(torch.zeros((1, 1, 16, 64), dtype=bf), torch.zeros((1, 1, 16, 64), dtype=bf))
    with pytest.raises(ValueError, match="CUDA"):
        gs.Batch(*(torch.zeros(2, dtype=torch.int32),) * 3, 1)
    with pytest.raises(ValueError, match="same length"):
        gs.adapters_batched_into([x], [], [], x, x, [])
    with pytest.raises(ValueError, match="CUDA"):
        gs._heads(torch.zeros((2, 4, 64), dtype=bf), 64, "q")
