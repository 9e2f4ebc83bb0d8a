"""No GPU needed: what the shared-prefix attention refuses before anything is launched."""
from tests.test_pool_refusals import P, _kv, _status, binding, ctx  # noqa: F401  (fixtures)


def _call(binding, ctx, ks=(2, 0), **kw):
    a = dict(q=P, spec=P, h=None if ks is None else binding.host_i32(ks), B=2, prefix=32, max_ctx=60, kv=_kv(binding), layer=0, out=P, ws=0x2000, n=1 << 40)
    a.update(kw)
    binding.mn_prefix_attention(ctx, a["q"], a["spec"], a["h"], a["B"], a["prefix"], a["max_ctx"], a["kv"], a["layer"], a["out"], a["ws"], a["n"])


def test_pointers_and_counts(binding, ctx):  # noqa: F811
    E = binding
    for key in ("q", "spec", "out", "ws"):
        assert _status(E, lambda: _call(E, ctx, **{key: None})) == E.MN_ENULL
    assert _status(E, lambda: _call(E, ctx, ks=None)) == E.MN_ENULL
    for bad in (dict(B=-1), dict(B=E.MN_MAX_BATCH + 1), dict(max_ctx=-1), dict(ks=(2, -1)), dict(layer=1), dict(layer=-1), dict(q=P + 2), dict(out=P + 8)):
        assert _status(E, lambda: _call(E, ctx, **bad)) == E.MN_EINVAL
    _call(E, ctx, B=0, q=None)
    assert E.lib.mn_prefix_attention(None, P, P, None, 0, 0, 0, None, 0, P, P, 0, None, None) == E.MN_ENULL


def test_prefix_contexts_and_cache(binding, ctx):  # noqa: F811
    E = binding
    for bad in (dict(prefix=-16), dict(prefix=20), dict(prefix=64, max_ctx=64), dict(prefix=48, max_ctx=50)):
        assert _status(E, lambda: _call(E, ctx, **bad)) == E.MN_EINVAL
    assert _status(E, lambda: _call(E, ctx, max_ctx=65)) == E.MN_ECAPACITY                       # 4 blocks of 16
    assert _status(E, lambda: _call(E, ctx, max_ctx=129, kv=_kv(E, width=99))) == E.MN_ECAPACITY  # max_pos
    assert _status(E, lambda: _call(E, ctx, kv=_kv(E, bt=None))) == E.MN_ENULL
    assert _status(E, lambda: _call(E, ctx, kv=_kv(E, nb=0))) == E.MN_EINVAL


def test_workspace(binding, ctx):  # noqa: F811
    E = binding
    need = E.mn_prefix_workspace_bytes(ctx, 2, 4, 32, 60)
    assert need > 0
    assert _status(E, lambda: _call(E, ctx, ws=0x2010)) == E.MN_EWORKSPACE
    assert _status(E, lambda: _call(E, ctx, n=need - 1)) == E.MN_EWORKSPACE
    for bad in ((-1, 4, 32, 60), (2, -1, 32, 60), (2, 4, -1, 60), (2, 4, 32, 31), (E.MN_MAX_BATCH + 1, 4, 32, 60)):
        assert E.mn_prefix_workspace_bytes(ctx, *bad) == 0
    # a workspace for more rows, sequences or longer contexts serves what is smaller
    sizes = [E.mn_prefix_workspace_bytes(ctx, 64, m, 4096, 9000) for m in (1, 5, 16, 33, 64, 100, 500, 3000, 20000)]
    assert sizes == sorted(sizes)
    sizes = [E.mn_prefix_workspace_bytes(ctx, b, 4096, 4096, 9000) for b in (1, 3, 64, 1000, 4096)]
    assert sizes == sorted(sizes)
    sizes = [E.mn_prefix_workspace_bytes(ctx, 8, 72, 4096, c) for c in (4097, 4200, 4353, 5000, 100000)]
    assert sizes == sorted(sizes)


def test_blocks_whose_pages_pass_32_bits(binding, ctx):  # noqa: F811
    from tests.test_prompt_refusals import _call as prompt
    E, bs = binding, 1 << 24                                        # of heads of 128: 2^31 elements
    assert _status(E, lambda: _call(E, ctx, prefix=0, kv=_kv(E, bs=bs))) == E.MN_EUNSUPPORTED
    assert _status(E, lambda: prompt(E, ctx, kv=_kv(E, bs=bs))) == E.MN_EUNSUPPORTED
