"""No GPU needed: what the prompt attention refuses before anything is launched."""
import pytest

from tests.test_abi import _desc, _weights
from tests.test_pool_refusals import P, _kv, _status, binding, ctx  # noqa: F401  (fixtures)


def _call(binding, ctx, rows=(0, 3, 3, 10), **kw):
    a = dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, dev=P, h=None if rows is None else binding.host_i32(rows), B=3, out=P, kv=None, layer=0)
    a.update(kw)
    binding.mn_prompt_attention(ctx, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["dev"], a["h"], a["B"], a["out"], a["kv"], a["layer"])


def test_pointers_counts_and_offsets(binding, ctx):  # noqa: F811
    for key in ("q", "k", "v", "dev", "out"):
        assert _status(binding, lambda: _call(binding, ctx, **{key: None})) == binding.MN_ENULL
    assert _status(binding, lambda: _call(binding, ctx, rows=None)) == binding.MN_ENULL
    for B in (-1, binding.MN_MAX_BATCH + 1):
        assert _status(binding, lambda: _call(binding, ctx, B=B)) == binding.MN_EINVAL
    for rows in ((-1, 3, 3, 10), (0, 3, 2, 10), (0, 3, 3, (1 << 20) + 1), (5, 3, 8, 10)):
        assert _status(binding, lambda: _call(binding, ctx, rows=rows)) == binding.MN_EINVAL
    _call(binding, ctx, B=0, q=None, rows=None)                      # nothing to do
    _call(binding, ctx, rows=(4, 4, 4, 4))
    assert binding.lib.mn_prompt_attention(None, P, 256, P, 128, P, 128, P, None, 0, None, 0, P, None, None) == binding.MN_ENULL


def test_strides_and_alignment(binding, ctx):  # noqa: F811
    for key, short, odd in (("qs", 248, 260), ("ks", 120, 132), ("vs", 0, 129)):
        assert _status(binding, lambda: _call(binding, ctx, **{key: short})) == binding.MN_EINVAL
        assert _status(binding, lambda: _call(binding, ctx, **{key: odd})) == binding.MN_EINVAL
    for key in ("q", "k", "v", "out"):
        assert _status(binding, lambda: _call(binding, ctx, **{key: P + 8})) == binding.MN_EINVAL


def test_the_cache_is_checked(binding, ctx):  # noqa: F811
    assert _status(binding, lambda: _call(binding, ctx, kv=_kv(binding, bt=None))) == binding.MN_ENULL
    assert _status(binding, lambda: _call(binding, ctx, kv=_kv(binding, bs=0))) == binding.MN_EINVAL
    assert _status(binding, lambda: _call(binding, ctx, kv=_kv(binding), layer=1)) == binding.MN_EINVAL
    assert _status(binding, lambda: _call(binding, ctx, rows=(0, 3, 3, 68), kv=_kv(binding))) == binding.MN_ECAPACITY   # 65 tokens in 4 blocks
    assert _status(binding, lambda: _call(binding, ctx, rows=(0, 0, 0, 129), kv=_kv(binding, width=99))) == binding.MN_ECAPACITY   # max_pos


@pytest.fixture(scope="module")
def wide(binding):  # noqa: F811
    """512 heads of 8."""
    d = _desc(binding, d_model=4096, n_heads=512, n_kv_heads=512, head_dim=8, max_pos=1 << 21)
    w, keep = _weights(binding)
    c = binding.mn_create(d, w)
    yield c
    binding.mn_destroy(c)


def test_more_workgroups_than_a_launch_holds(binding, wide):  # noqa: F811
    kw = dict(qs=4096, ks=4096, vs=4096, B=1)
    assert _status(binding, lambda: _call(binding, wide, rows=(0, 1 << 20), **kw)) == binding.MN_EUNSUPPORTED
    assert _status(binding, lambda: _call(binding, wide, rows=(0, (1 << 19) + 1), **kw)) == binding.MN_EUNSUPPORTED


def test_more_workgroups_than_a_launch_holds_behind_a_prefix(binding, wide):  # noqa: F811
    ks, kv = binding.host_i32([255] * 4096), _kv(binding, width=1 << 16, nb=1 << 16)
    for prefix in (0, 16):
        assert _status(binding, lambda: binding.mn_prefix_attention(wide, P, P, ks, 4096, prefix, 100000, kv, 0, P, 0x2000, 1 << 60)) == binding.MN_EUNSUPPORTED
