"""The 8-bit paged cache without a GPU: what its entry points refuse before they touch a device, the sizes that they ask for, the
Python handle, and the oracle against what is known of the formats."""
import ctypes

import numpy as np
import pytest
import torch

import kv8_oracle as o
import paper_2605_02905_b200 as eosq

OK, INVALID, UNSUPPORTED, SMALL = eosq.EOSQ_OK, eosq.EOSQ_ERR_INVALID_ARG, eosq.EOSQ_ERR_UNSUPPORTED, eosq.EOSQ_ERR_BUFFER_TOO_SMALL
P = 1 << 20            # an address that is never followed: every call below is refused, or has nothing to do
CTX = 1 << 21


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2605_02905_b200 import build
    build.build()


def _cache(**kw):
    c = eosq._Kv8Struct()
    for name in ("k", "v", "k_scale", "v_scale", "table", "lengths", "refs", "flags"):
        setattr(c, name, P)
    for name, value in dict(layers=2, num_pages=64, kv_heads=3, page_size=32, d=128, format=0, max_seqs=8, max_pages=10).items():
        setattr(c, name, value)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def _calls(c, *, ctx=CTX, n=2, lists=P, layer=0, dtype=0, rows=P, stride=1024, total=4, most=2, G=2, scale=0.1, causal=1, window=0, lse=P, ws=P, wsb=1 << 40):
    L, a = eosq.lib(), ctypes.pointer(c)   # (a pointer keeps its object)
    return {
        "reserve": lambda: L.eosq_kv8_reserve(ctx, a, lists, lists, n, lists, None),
        "store": lambda: L.eosq_kv8_store(ctx, a, layer, rows, rows, dtype, total, stride, 128, stride, 128, lists, lists, lists, n, most, None),
        "attend": lambda: L.eosq_kv8_attend(ctx, a, layer, rows, dtype, total, stride, 128, lists, lists, n, most, G, scale, causal, window, rows, stride, 128,
                                            lse, ws, wsb, None),
        "fork": lambda: L.eosq_kv8_fork(ctx, a, lists, lists, n, ws, wsb, None),
        "free": lambda: L.eosq_kv8_free(ctx, a, lists, n, None),
        "compact": lambda: L.eosq_kv8_compact(ctx, a, lists, ws, wsb, None),
        "copy_pages": lambda: L.eosq_kv8_copy_pages(ctx, a, a, lists, lists, n, None),
        "check": lambda: L.eosq_kv8_check(ctx, a, None, None),
    }


ALL = list(_calls(_cache()))


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("bad,want", [
    (dict(layers=0), INVALID), (dict(num_pages=-1), INVALID), (dict(kv_heads=0), INVALID), (dict(max_seqs=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(k=None), INVALID), (dict(flags=None), INVALID), (dict(k=P + 8), INVALID), (dict(v_scale=P + 2), INVALID), (dict(table=P + 1), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(d=256), UNSUPPORTED),
    (dict(format=2), UNSUPPORTED), (dict(max_seqs=8193), UNSUPPORTED), (dict(num_pages=(1 << 20) + 1), UNSUPPORTED),
    (dict(num_pages=1 << 20, kv_heads=64), UNSUPPORTED), (dict(max_pages=1 << 26), UNSUPPORTED),
])
def test_a_cache_that_is_none(name, bad, want):
    assert _calls(_cache(**bad))[name]() == want


@pytest.mark.parametrize("name", ALL)
def test_no_context(name):
    assert _calls(_cache(), ctx=None)[name]() == INVALID


@pytest.mark.parametrize("name,bad,want", [
    (name, dict(lists=None), INVALID) for name in ("reserve", "store", "attend", "fork", "free", "compact", "copy_pages")] + [
    (name, dict(lists=P + 2), INVALID) for name in ("reserve", "store", "attend", "fork", "free", "compact", "copy_pages")] + [
    (name, dict(n=-1), INVALID) for name in ("reserve", "store", "attend", "fork", "free", "copy_pages")] + [
    (name, dict(n=0), OK) for name in ("reserve", "store", "attend", "fork", "free", "copy_pages")] + [
    (name, dict(n=8193), UNSUPPORTED) for name in ("reserve", "store", "attend", "fork", "free")] + [
    (name, dict(wsb=255), SMALL) for name in ("attend", "fork", "compact")] + [
    (name, dict(ws=None), INVALID) for name in ("attend", "fork", "compact")] + [
    (name, dict(ws=P + 128), INVALID) for name in ("attend", "fork", "compact")] + [
    (name, b, INVALID) for name in ("store", "attend") for b in (dict(rows=None), dict(rows=P + 8), dict(stride=1025), dict(stride=-1024), dict(layer=2), dict(layer=-1),
                                                                 dict(total=-1), dict(most=-1), dict(dtype=3))] + [
    ("store", dict(total=0), OK), ("store", dict(most=0), OK), ("store", dict(dtype=1, stride=1026), INVALID), ("attend", dict(total=0), OK), ("attend", dict(most=0), OK),
    ("attend", dict(dtype=1), INVALID), ("attend", dict(G=0), INVALID), ("attend", dict(window=-1), INVALID), ("attend", dict(window=5, causal=0), INVALID),
    ("attend", dict(scale=float("nan")), INVALID), ("attend", dict(scale=float("inf")), INVALID), ("attend", dict(lse=P + 2), INVALID),
    ("attend", dict(total=(1 << 31) - 1, most=1, G=64), UNSUPPORTED), ("store", dict(total=1 << 31), UNSUPPORTED), ("attend", dict(total=1 << 31), UNSUPPORTED), ("copy_pages", dict(n=(1 << 20) + 1), UNSUPPORTED),
])
def test_arguments_that_are_refused(name, bad, want):
    assert _calls(_cache(), **bad)[name]() == want


def test_pools_of_two_kinds():
    a = _cache()
    for other in (_cache(page_size=64), _cache(d=64), _cache(format=1), _cache(kv_heads=4), _cache(layers=1)):
        assert eosq.lib().eosq_kv8_copy_pages(CTX, ctypes.pointer(a), ctypes.pointer(other), P, P, 1, None) == INVALID


def test_workspace_sizes():
    size = lambda rows=0, **kw: eosq.lib().eosq_kv8_workspace_bytes(ctypes.pointer(_cache(**kw)), rows)
    assert size() >= 4 * (64 + 64) and size() % 256 == 0
    assert size(num_pages=100000) >= 4 * 100064 and size(max_seqs=8192) >= 8 * 8192
    assert size(8) >= 4 * 8193 and size(8) % 256 == 0 and size(4096) >= size(17)
    assert size(-1) == 0 and size(d=96) == 0
    # what a call asks for is what this names
    c, need = _cache(), size(4)
    assert _calls(c, wsb=need - 256)["attend"]() == SMALL


def test_the_handle():
    c = eosq.Kv8Cache.allocate(2, 5, 3, 16, 64, eosq.EOSQ_KV_E4M3, 4, 6, device="cpu")
    assert (c.layers, c.num_pages, c.kv_heads, c.page_size, c.d, c.max_seqs, c.max_pages, c.format) == (2, 5, 3, 16, 64, 4, 6, 1)
    assert bool((c.table == -1).all()) and int(c.lengths.sum()) == 0 and int(c.refs.sum()) == 0 and int(c.flags) == 0
    with pytest.raises(AttributeError):
        c.k = c.v
    fields = {name: getattr(c, name) for name in ("k", "v", "k_scale", "v_scale", "table", "lengths", "refs")}
    for name, bad in (("v", c.k[:1]), ("k_scale", c.k_scale.double()), ("table", c.table.t()), ("lengths", c.lengths[:3]), ("refs", c.refs.long())):
        with pytest.raises(ValueError):
            eosq.Kv8Cache(**{**fields, name: bad}, format=0)
    class NoContext:
        _h = None
    q = torch.zeros(2, 6, 64, dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    for args in ((q[:, :, :32], i[:1], i), (q[:, :5], i[:1], i), (q, i[:1].long(), i), (q, i[:1], i[:1])):
        with pytest.raises(ValueError):
            eosq.eosq_kv8_attend(NoContext, c, 0, *args, 2)
    for call in (lambda: eosq.eosq_kv8_free(NoContext, c, i), lambda: eosq.eosq_kv8_check(NoContext, c), lambda: eosq.eosq_kv8_compact(NoContext, c),
                 lambda: eosq.eosq_kv8_attend(NoContext, c, 0, q, i[:1], i, 2)):
        with pytest.raises(ValueError, match="not the current CUDA device"):
            call()
    with pytest.raises(TypeError):
        eosq.eosq_kv8_store(NoContext, c, 0, q.double()[:, :3], q.double()[:, :3], i[:1], i[:1], i, 2)


def test_the_oracle_knows_the_formats():
    """e4m3 against torch's conversion; halves go to even codes; scales at the borders."""
    every = torch.arange(256, dtype=torch.uint8)
    t = every.view(torch.float8_e4m3fn).double().numpy()
    known = ~np.isnan(t)
    assert np.array_equal(o.E4M3_VALUES[known], t[known]) and int(known.sum()) == 254
    x = torch.cat([torch.linspace(-450, 450, 20011), torch.randn(20000) * 2.0 ** torch.randint(-14, 8, (20000,))]).clamp(-448, 448)
    assert np.array_equal(o.decode(1, o.encode(1, x.double().numpy())), x.to(torch.float8_e4m3fn).double().numpy())
    assert np.array_equal(o.encode(1, o.E4M3_VALUES[:127]), np.arange(127)) and np.array_equal(o.encode(1, np.array([500.0, -np.inf, np.nan])), [126, 254, 0])
    assert o.encode(0, np.array([0.5, 1.5, -2.5, 126.5, 127.49, -300.0, np.nan, np.inf])).view(np.int8).tolist() == [0, 2, -2, 126, 127, -127, 0, 127]
    assert o.scale_of(1, 448.0) == 1.0 and o.scale_of(1, np.nextafter(448.0, 500)) == 2.0 and o.scale_of(1, 224.0) == 0.5 and o.scale_of(1, 0.0) == 2.0 ** -64
    assert o.scale_of(0, 127.0) == 1.0 and o.scale_of(0, 0.0) == 2.0 ** -64 and o.scale_of(0, 3e38) == 2.0 ** 64


def test_a_padded_list_to_fork():
    """A call's list may be longer than the cache has sequences (entries of -1 are padding), in fork as in the other calls: up to the workspace, nothing refuses it."""
    c = _cache(max_seqs=8)
    for n in (9, 100, 8192):
        assert _calls(c, n=n, wsb=255)["fork"]() == SMALL
    need = eosq.lib().eosq_kv8_workspace_bytes(ctypes.pointer(c), 0)
    assert need >= 8 * 8192 and _calls(c, n=9, wsb=need - 256)["fork"]() == SMALL
