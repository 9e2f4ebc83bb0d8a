"""No GPU needed: what the page pool's entry points refuse before anything is launched."""
import ctypes as C

import pytest

from tests.test_abi import _desc, _weights

P = 0x1000          # never dereferenced


@pytest.fixture(scope="module")
def binding():
    from paper_2402_15678_amd import binding
    return binding


@pytest.fixture(scope="module")
def ctx(binding):
    w, keep = _weights(binding)
    c = binding.mn_create(_desc(binding), w)
    yield c
    binding.mn_destroy(c)


def _kv(binding, **kw):
    arr = binding.ptr_array([P])
    a = dict(k=C.cast(arr, C.POINTER(C.c_void_p)), v=C.cast(arr, C.POINTER(C.c_void_p)), bs=16, nb=8, width=4, bt=P, ctx=P)
    a.update(kw)
    kv = binding.KV(a["k"], a["v"], a["bs"], a["nb"], a["width"], a["bt"], a["ctx"])
    kv.keep = arr
    return kv


def _pool(binding, **kw):
    a = dict(bt=P, refs=P, held=P, slots=4)
    a.update(kw)
    return binding.Pool(a["bt"], a["refs"], a["held"], a["slots"])


def _status(binding, call):
    with pytest.raises(binding.MinionsError) as e:
        call()
    return e.value.status


def test_workspace_query(binding):
    assert binding.mn_kv_workspace_bytes(0, 4) == 0 and binding.mn_kv_workspace_bytes(8, 0) == 0
    assert binding.mn_kv_workspace_bytes(8, binding.MN_MAX_BATCH + 1) == 0
    assert binding.mn_kv_workspace_bytes(1000, 4) >= 4 * 4 * 1000


def test_every_call_checks_kv_and_pool(binding, ctx):
    ws, n = 0x2000, 1 << 20
    calls = [lambda kv, p: binding.mn_kv_reserve(ctx, kv, p, P, 2, ws, n), lambda kv, p: binding.mn_kv_fork(ctx, kv, p, P, P, 2),
             lambda kv, p: binding.mn_kv_free(ctx, kv, p, P, 2), lambda kv, p: binding.mn_kv_compact(ctx, kv, p, P, ws, n)]
    for call in calls:
        for bad in (dict(bt=None), dict(ctx=None)):
            assert _status(binding, lambda: call(_kv(binding, **bad), _pool(binding))) == binding.MN_ENULL
        for bad in (dict(bs=0), dict(nb=0), dict(width=-1)):
            assert _status(binding, lambda: call(_kv(binding, **bad), _pool(binding))) == binding.MN_EINVAL
        for bad in (dict(refs=None), dict(held=None), dict(bt=None)):
            assert _status(binding, lambda: call(_kv(binding), _pool(binding, **bad))) == binding.MN_ENULL
        for bad in (dict(bt=0x3000), dict(slots=0), dict(slots=binding.MN_MAX_BATCH + 1)):
            assert _status(binding, lambda: call(_kv(binding), _pool(binding, **bad))) == binding.MN_EINVAL


def test_counts_lists_and_workspaces(binding, ctx):
    kv, pool, E = _kv(binding), _pool(binding), binding
    for n in (-1, 5):
        assert _status(E, lambda: E.mn_kv_reserve(ctx, kv, pool, P, n, 0x2000, 1 << 20)) == E.MN_EINVAL
        assert _status(E, lambda: E.mn_kv_fork(ctx, kv, pool, P, P, n)) == E.MN_EINVAL
        assert _status(E, lambda: E.mn_kv_free(ctx, kv, pool, P, n)) == E.MN_EINVAL
    E.mn_kv_reserve(ctx, kv, pool, None, 0, 0x2000, 1 << 20)      # nothing to do: no launch
    E.mn_kv_fork(ctx, kv, pool, None, None, 0)
    E.mn_kv_free(None, kv, pool, None, 0)
    assert _status(E, lambda: E.mn_kv_reserve(ctx, kv, pool, None, 1, 0x2000, 1 << 20)) == E.MN_ENULL
    assert _status(E, lambda: E.mn_kv_fork(ctx, kv, pool, P, None, 1)) == E.MN_ENULL
    assert _status(E, lambda: E.mn_kv_free(ctx, kv, pool, None, 1)) == E.MN_ENULL
    need = E.mn_kv_workspace_bytes(8, 4)
    for call in (lambda ws, n: E.mn_kv_reserve(ctx, kv, pool, P, 1, ws, n), lambda ws, n: E.mn_kv_compact(ctx, kv, pool, None, ws, n)):
        assert _status(E, lambda: call(None, need)) == E.MN_ENULL
        assert _status(E, lambda: call(0x2010, need)) == E.MN_EWORKSPACE
        assert _status(E, lambda: call(0x2000, need - 1)) == E.MN_EWORKSPACE
    null = binding.ptr_array([None])
    layerless = _kv(binding, k=C.cast(null, C.POINTER(C.c_void_p)))
    assert _status(E, lambda: E.mn_kv_reserve(ctx, layerless, pool, P, 1, 0x2000, need)) == E.MN_ENULL
    assert _status(E, lambda: E.mn_kv_compact(ctx, _kv(binding, v=None), pool, None, 0x2000, need)) == E.MN_ENULL
    assert E.lib.mn_kv_reserve(None, None, None, None, 0, None, 0, None, None) == E.MN_ENULL
    assert E.lib.mn_kv_compact(None, None, None, None, None, 0, None, None) == E.MN_ENULL


def test_a_context_without_layers_needs_the_pages_of_layer_0(binding):
    w, keep = _weights(binding)
    c = binding.mn_create(_desc(binding, n_layers=0), w)
    need, none = binding.mn_kv_workspace_bytes(8, 4), C.cast(binding.ptr_array([None]), C.POINTER(C.c_void_p))
    for pages in (dict(k=none), dict(v=none)):
        assert _status(binding, lambda: binding.mn_kv_reserve(c, _kv(binding, **pages), _pool(binding), P, 1, 0x2000, need)) == binding.MN_ENULL
        assert _status(binding, lambda: binding.mn_kv_compact(c, _kv(binding, **pages), _pool(binding), None, 0x2000, need)) == binding.MN_ENULL
    binding.mn_destroy(c)


def test_numbers_of_blocks_beyond_what_the_plans_count(binding, ctx):
    E, need, most = binding, 1 << 40, (1 << 31) - 1
    assert E.mn_kv_workspace_bytes((1 << 30) + 1, 4) == 0 and E.mn_kv_workspace_bytes(most, 4) == 0
    for nb in ((1 << 30) + 1, most):
        assert _status(E, lambda: E.mn_kv_reserve(ctx, _kv(E, nb=nb), _pool(E), P, 1, 0x2000, need)) == E.MN_EUNSUPPORTED
        assert _status(E, lambda: E.mn_kv_compact(ctx, _kv(E, nb=nb), _pool(E), None, 0x2000, need)) == E.MN_EUNSUPPORTED
    # 4096 rows that may each ask for 2^19 blocks: their sum passes 32 bits
    wide, slots = _kv(E, nb=1 << 30, width=1 << 19), _pool(E, slots=4096)
    assert _status(E, lambda: E.mn_kv_reserve(ctx, wide, slots, P, 4096, 0x2000, need)) == E.MN_EUNSUPPORTED
