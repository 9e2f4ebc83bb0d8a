"""No GPU needed: what the calls of a bounded cache refuse before anything is launched."""
import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2402_15678_amd import harness, synth
from tests.test_abi import _desc, _weights
from tests.test_pool_refusals import P, _kv, _status, binding, ctx  # noqa: F401  (fixtures)

BIG = 1 << 40                                                        # a workspace that is never too small


@pytest.fixture(scope="module")
def wide(binding):  # noqa: F811
    """512 heads of 8."""
    w, keep = _weights(binding)
    c = binding.mn_create(_desc(binding, d_model=4096, n_heads=512, n_kv_heads=512, head_dim=8, max_pos=1 << 21), w)
    yield c
    binding.mn_destroy(c)


def _rule(binding, gains=(P, P), eps=1e-5, rot=128, pairs=(64,), base=10000.0, axes=None):  # noqa: F811
    return binding.RowRule(*gains, eps, rot, len(pairs) if axes is None else axes, (C.c_int * 4)(*pairs), base)


def _rows(binding, ctx, h=(2, 0, 4), **kw):  # noqa: F811
    a = dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, f32=0, rule=_rule(binding), pos=P, spec=P, h=None if h is None else binding.host_i32(h), B=3, kv=_kv(binding),
             layer=0, q_out=P, k_out=None, v_out=None)
    a.update(kw)
    binding.mn_qk_norm_rope(ctx, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["f32"], a["rule"], a["pos"], a["spec"], a["h"], a["B"], a["kv"], a["layer"],
                            a["q_out"], a["k_out"], a["v_out"])


def test_rows_pointers_rules_and_shapes(binding, ctx):  # noqa: F811
    refused = lambda status, **kw: _status(binding, lambda: _rows(binding, ctx, **kw)) == status  # noqa: E731
    for key in ("q", "k", "v", "rule", "pos", "spec", "h"):
        assert refused(binding.MN_ENULL, **{key: None}), key
    for B in (-1, binding.MN_MAX_BATCH + 1):
        assert refused(binding.MN_EINVAL, B=B)
    for rot, pairs in ((132, (66,)), (136, (68,)), (-8, (0,)), (4, (2,)), (128, (-1,)), (128, (65, -1))):
        assert refused(binding.MN_EINVAL, rule=_rule(binding, rot=rot, pairs=pairs)), rot
    for axes in (0, 5):
        assert refused(binding.MN_EINVAL, rule=_rule(binding, axes=axes))
    for pairs in ((63,), (32, 33), (16, 16, 16), (0, 0, 0, 0)):
        assert refused(binding.MN_ESHAPE, rule=_rule(binding, pairs=pairs))
    for base in (0.0, -1.0, float("nan"), float("inf")):
        assert refused(binding.MN_EINVAL, rule=_rule(binding, base=base))
    for eps in (-1e-9, float("nan"), float("inf")):
        assert refused(binding.MN_EINVAL, rule=_rule(binding, eps=eps))
    for key, short, odd in (("qs", 248, 260), ("ks", 120, 132), ("vs", 0, 129)):
        assert refused(binding.MN_EINVAL, **{key: short}) and refused(binding.MN_EINVAL, **{key: odd})
    for key in ("q", "k", "v", "q_out", "k_out", "v_out"):
        assert refused(binding.MN_EINVAL, **{key: P + 8}), key
    for h in ((-1, 0, 4), (0, 1 << 20, 0)):
        assert refused(binding.MN_EINVAL, h=h)
    assert refused(binding.MN_ENULL, kv=_kv(binding, bt=None)) and refused(binding.MN_EINVAL, kv=_kv(binding, bs=0)) and refused(binding.MN_EINVAL, layer=1)
    assert refused(binding.MN_ECAPACITY, h=(64, 0, 0))                # 65 rows in 4 blocks of 16
    assert refused(binding.MN_EUNSUPPORTED, kv=_kv(binding, width=1 << 26, nb=1 << 26))
    _rows(binding, ctx, B=0, q=None, h=None)                          # nothing to do
    _rows(binding, ctx, kv=None, q_out=None, q=None, k=None, v=None, spec=None, qs=0, ks=0, vs=0)
    assert binding.lib.mn_qk_norm_rope(None, P, 256, P, 128, P, 128, 0, None, P, P, None, 0, None, 0, P, None, None, None, None) == binding.MN_ENULL


def _window(binding, ctx, h=(2, 0, 4), **kw):  # noqa: F811
    a = dict(q=P, spec=P, h=None if h is None else binding.host_i32(h), B=3, window=8, sinks=2, max_ctx=40, kv=_kv(binding), layer=0, out=P, stats=P, ws=0x2000, wsb=BIG)
    a.update(kw)
    binding.mn_window_attention(ctx, a["q"], a["spec"], a["h"], a["B"], a["window"], a["sinks"], a["max_ctx"], a["kv"], a["layer"], a["out"], a["stats"], a["ws"], a["wsb"])


def test_windows(binding, ctx, wide):  # noqa: F811
    refused = lambda status, **kw: _status(binding, lambda: _window(binding, ctx, **kw)) == status  # noqa: E731
    for key in ("q", "spec", "h", "out", "ws"):
        assert refused(binding.MN_ENULL, **{key: None}), key
    for kw in (dict(B=-1), dict(B=binding.MN_MAX_BATCH + 1), dict(window=0), dict(window=-3), dict(sinks=-1), dict(max_ctx=-1), dict(max_ctx=4), dict(q=P + 8), dict(out=P + 4),
               dict(stats=P + 4), dict(layer=1), dict(layer=-1), dict(h=(-1, 0, 1)), dict(kv=_kv(binding, bs=0))):
        assert refused(binding.MN_EINVAL, **kw), kw
    assert refused(binding.MN_ENULL, kv=_kv(binding, bt=None))
    assert refused(binding.MN_ECAPACITY, max_ctx=65) and refused(binding.MN_ECAPACITY, max_ctx=129, kv=_kv(binding, width=99))   # the table, max_pos
    assert refused(binding.MN_EWORKSPACE, ws=0x2010) and refused(binding.MN_EWORKSPACE, wsb=100)
    need = binding.mn_window_workspace_bytes(ctx, 3, 9)
    assert need > 0 and refused(binding.MN_EWORKSPACE, wsb=need - 1)
    assert binding.mn_window_workspace_bytes(ctx, -1, 9) == 0 and binding.mn_window_workspace_bytes(ctx, 3, -1) == 0 and binding.mn_window_workspace_bytes(None, 3, 9) == 0
    # a workspace for the largest batch serves every smaller one
    sizes = [[binding.mn_window_workspace_bytes(ctx, b, m) for m in (1, 9, 100, 5000, 1 << 20)] for b in (1, 3, 64, 65, 4096)]
    assert all(x <= y for r in sizes for x, y in zip(r, r[1:])) and all(x <= y for r, s in zip(sizes, sizes[1:]) for x, y in zip(r, s))
    _window(binding, ctx, B=0, q=None, h=None)
    assert _status(binding, lambda: _window(binding, wide, h=((1 << 20) - 1,), B=1, max_ctx=1 << 20, kv=_kv(binding, width=1 << 16, nb=1 << 16))) == binding.MN_EUNSUPPORTED
    assert binding.lib.mn_window_attention(None, P, P, None, 0, 8, 2, 40, None, 0, P, None, P, BIG, None, None) == binding.MN_ENULL


def _ledger(binding, mass=P, born=P, seqs=8, width=64):  # noqa: F811
    return binding.Ledger(mass, born, seqs, width)


def _weigh(binding, ctx, h=(2, 0, 4), **kw):  # noqa: F811
    a = dict(q=P, stats=P, spec=P, h=None if h is None else binding.host_i32(h), B=3, n_out=None, seen=None, max_ctx=40, kv=_kv(binding), layer=0, ledger=_ledger(binding))
    a.update(kw)
    binding.mn_kv_weigh(ctx, a["q"], a["stats"], a["spec"], a["h"], a["B"], a["n_out"], a["seen"], a["max_ctx"], a["kv"], a["layer"], a["ledger"])


def test_weights(binding, ctx, wide):  # noqa: F811
    refused = lambda status, **kw: _status(binding, lambda: _weigh(binding, ctx, **kw)) == status  # noqa: E731
    for key in ("q", "stats", "spec", "h", "ledger"):
        assert refused(binding.MN_ENULL, **{key: None}), key
    for kw in (dict(mass=None), dict(born=None)):
        assert refused(binding.MN_ENULL, ledger=_ledger(binding, **kw))
    for kw in (dict(width=0), dict(width=1 << 28), dict(seqs=0), dict(seqs=2), dict(seqs=binding.MN_MAX_BATCH + 1)):
        assert refused(binding.MN_EINVAL, ledger=_ledger(binding, **kw)), kw
    for kw in (dict(B=-1), dict(B=binding.MN_MAX_BATCH + 1), dict(max_ctx=-1), dict(q=P + 8), dict(stats=P + 4), dict(layer=1), dict(h=(-1, 0, 1)), dict(kv=_kv(binding, bs=0))):
        assert refused(binding.MN_EINVAL, **kw), kw
    assert refused(binding.MN_ECAPACITY, ledger=_ledger(binding, width=39)) and refused(binding.MN_ECAPACITY, max_ctx=65)
    _weigh(binding, ctx, B=0, q=None, h=None)
    kv = _kv(binding, width=1 << 17, nb=1 << 17)
    assert _status(binding, lambda: _weigh(binding, wide, h=[0] * 4096, B=4096, max_ctx=1 << 20, kv=kv, ledger=_ledger(binding, seqs=4096, width=1 << 20))) == binding.MN_EUNSUPPORTED
    assert binding.lib.mn_kv_weigh(None, P, P, P, None, 0, None, None, 40, None, 0, None, None, None) == binding.MN_ENULL


def _evict(binding, ctx, **kw):  # noqa: F811
    a = dict(kv=_kv(binding), pool=binding.Pool(P, P, P, 8), keep=P, B=3, sinks=2, recent=4, ledger=_ledger(binding), ws=0x2000, wsb=BIG)
    a.update(kw)
    binding.mn_kv_evict(ctx, a["kv"], a["pool"], a["keep"], a["B"], a["sinks"], a["recent"], a["ledger"], a["ws"], a["wsb"])


def test_evictions(binding, ctx, wide):  # noqa: F811
    refused = lambda status, **kw: _status(binding, lambda: _evict(binding, ctx, **kw)) == status  # noqa: E731
    for key in ("keep", "ledger", "ws"):
        assert refused(binding.MN_ENULL, **{key: None}), key
    for kw in (dict(B=-1), dict(B=9), dict(sinks=-1), dict(recent=-1), dict(ledger=_ledger(binding, seqs=7)), dict(ledger=_ledger(binding, width=0)),
               dict(pool=binding.Pool(P + 64, P, P, 8)), dict(pool=binding.Pool(P, P, P, 0))):
        assert refused(binding.MN_EINVAL, **kw), kw
    for pool in (binding.Pool(P, None, P, 8), binding.Pool(P, P, None, 8)):
        assert refused(binding.MN_ENULL, pool=pool)
    assert refused(binding.MN_EWORKSPACE, ws=0x2010) and refused(binding.MN_EWORKSPACE, wsb=binding.mn_evict_workspace_bytes(ctx, 3, 64) - 1)
    assert binding.mn_evict_workspace_bytes(ctx, 3, 0) == 0 and binding.mn_evict_workspace_bytes(ctx, -1, 64) == 0 and binding.mn_evict_workspace_bytes(None, 3, 64) == 0
    _evict(binding, ctx, B=0, keep=None)
    assert binding.lib.mn_kv_evict(None, None, None, P, 0, 2, 4, None, P, BIG, None, None) == binding.MN_ENULL


@pytest.mark.parametrize("dtype,right", [(synth.DT_BF16, torch.float16), (synth.DT_F32, torch.float32)])
def test_rows_of_another_type_or_shape_are_refused(dtype, right, monkeypatch):
    """The calls themselves could not tell."""
    d = synth.ModelDesc(synth.ARCH_LLAMA, dtype, 1, 128, 2, 2, 64, 128, 8, 64)
    model, calls = SimpleNamespace(desc=d, ctx=None), []
    for name in ("mn_qk_norm_rope", "mn_window_attention", "mn_kv_weigh"):
        monkeypatch.setattr(harness.B, name, lambda *a, name=name: calls.append(name))
    monkeypatch.setattr(harness, "stream_ptr", lambda: 0)
    rule, spec = harness.RowRule(64, [32]), torch.tensor([2], dtype=torch.int32)
    new = lambda t, *s: torch.zeros(s, dtype=t)  # noqa: E731
    pos = torch.zeros((1, 3), dtype=torch.int32)

    def rows(t=right, out=right, heads=2, place=pos, length=(2,)):
        x = [new(t, 3, heads, 64) for _ in range(3)]
        harness.qk_norm_rope(model, *x, rule, place, spec, length, new(out, 3, 128))
    rows()
    rows(t=torch.float32)
    ses = harness.WindowSession.__new__(harness.WindowSession)
    ses.model, ses.kv, ses.max_q, ses.max_ctx, ses.window, ses.sinks, ses.ws_bytes = model, SimpleNamespace(c=None), 3, 32, 8, 0, 0
    ses.workspace = ses.dev_status = torch.zeros(1, dtype=torch.int32)
    ses.attention(new(right, 3, 2, 64), spec, [2], new(right, 3, 128), stats=new(torch.float32, 3, 2, 2))
    ledger = harness.KVLedger(model, SimpleNamespace(c=None), new(torch.float32, 1, 1, 2, 32), new(torch.int32, 1, 1, 2, 32))
    ledger.weigh(new(right, 3, 2, 64), new(torch.float32, 3, 2, 2), spec, [2], 0, 32)
    assert calls == ["mn_qk_norm_rope"] * 2 + ["mn_window_attention", "mn_kv_weigh"]
    wrong = sorted({torch.float16, torch.float32, torch.bfloat16} - {right}, key=str)
    for t in wrong:
        for call in (lambda: rows(out=t), lambda: ses.attention(new(t, 3, 2, 64), spec, [2], new(right, 3, 128)), lambda: ses.attention(new(right, 3, 2, 64), spec, [2], new(t, 3, 128)),
                     lambda: ledger.weigh(new(t, 3, 2, 64), new(torch.float32, 3, 2, 2), spec, [2], 0, 32)):
            with pytest.raises(AssertionError):
                call()
    for call in (lambda: rows(t=torch.bfloat16), lambda: rows(heads=1), lambda: rows(length=(1,)), lambda: rows(place=pos.float()), lambda: rows(place=pos[:, :2]),
                 lambda: ses.attention(new(right, 3, 2, 64), spec, [2], new(right, 3, 128), stats=new(right, 3, 2, 2).half()), lambda: ses.attention(new(right, 3, 2, 64), spec, [3], new(right, 3, 128)),
                 lambda: ledger.weigh(new(right, 3, 2, 64), new(torch.float16, 3, 2, 2), spec, [2], 0, 32),
                 lambda: harness.KVLedger(model, None, new(torch.float32, 1, 1, 3, 32), new(torch.int32, 1, 1, 3, 32)),
                 lambda: harness.KVLedger(model, None, new(torch.float32, 1, 1, 2, 32), new(torch.int32, 1, 1, 2, 31))):
        with pytest.raises(AssertionError):
            call()


def test_too_few_rows_and_numbers_of_another_type_or_device_are_refused(monkeypatch):
    """The library gets addresses: rows that are not there would be read, 64-bit numbers taken as pairs, a host's address as the device's."""
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16, 1, 128, 2, 2, 64, 128, 8, 64)
    model, calls = SimpleNamespace(desc=d, ctx=None), []

    class Far(torch.Tensor):
        def get_device(self):
            return 3
    for name in ("mn_qk_norm_rope", "mn_window_attention", "mn_kv_weigh", "mn_kv_evict"):
        monkeypatch.setattr(harness.B, name, lambda *a, name=name: calls.append(name))
    monkeypatch.setattr(harness, "stream_ptr", lambda: 0)
    half, whole = torch.float16, torch.float32
    new = lambda t, *s, far=False: torch.zeros(s, dtype=t).as_subclass(Far if far else torch.Tensor)  # noqa: E731
    i32 = lambda n, t=torch.int32, far=False: torch.zeros(n, dtype=t).as_subclass(Far if far else torch.Tensor)  # noqa: E731
    ses = harness.WindowSession.__new__(harness.WindowSession)
    ses.model, ses.kv, ses.max_q, ses.max_ctx, ses.window, ses.sinks, ses.ws_bytes = model, SimpleNamespace(c=None), 3, 32, 8, 0, 0
    ses.workspace = ses.dev_status = torch.zeros(1, dtype=torch.int32)
    ledger = harness.KVLedger(model, SimpleNamespace(c=None), new(whole, 1, 2, 2, 32), i32((1, 2, 2, 32)))
    pool = harness.KVPool.__new__(harness.KVPool)
    pool.model, pool.kv, pool.c, pool.dev_status = model, SimpleNamespace(c=None), None, i32(1)

    def rows(gain=64, spec=i32(2), pos=i32((1, 5)), k=False, out=False):
        rule = harness.RowRule(64, [32], 10000.0, new(whole, 64), new(whole, gain))
        harness.qk_norm_rope(model, new(half, 5, 2, 64), new(half, 5, 2, 64, far=k), new(half, 5, 2, 64), rule, pos, spec, [2, 1], new(half, 5, 128, far=out))

    def window(n=5, m=5, k=5, spec=i32(2), q=False, stats=False):
        ses.attention(new(half, n, 2, 64, far=q), spec, [2, 1], new(half, m, 128), stats=new(whole, k, 2, 2, far=stats))

    def weigh(n=5, k=5, spec=i32(2), n_out=None, seen=None, q=False, stats=False):
        ledger.weigh(new(half, n, 2, 64, far=q), new(whole, k, 2, 2, far=stats), spec, [2, 1], 0, 32, n_out, seen)

    def evict(keep):
        pool.evict(keep, 1, 1, ledger)
    rows()
    window()
    window(n=6, m=7, k=8)                                            # (buffers of a larger batch)
    weigh(n_out=i32(2), seen=i32(3))
    evict(i32(2))
    evict(i32(0))
    assert calls == ["mn_qk_norm_rope"] + ["mn_window_attention"] * 2 + ["mn_kv_weigh"] + ["mn_kv_evict"] * 2
    wrong = (i32(1), i32(2, torch.int64), i32(2, whole), i32(4)[::2], i32(2, far=True))
    bad = [lambda s=s, c=c: c(spec=s) for s in wrong for c in (rows, window, weigh)] + [lambda s=s, k=k: weigh(**{k: s}) for s in wrong for k in ("n_out", "seen")]
    bad += [lambda s=s: evict(s) for s in wrong[1:]]
    bad += [lambda kw=kw: rows(**kw) for kw in (dict(gain=32), dict(gain=128), dict(pos=i32((1, 5), far=True)), dict(k=True), dict(out=True))]
    bad += [lambda kw=kw: window(**kw) for kw in (dict(n=4), dict(m=4), dict(k=4), dict(q=True), dict(stats=True))]
    bad += [lambda kw=kw: weigh(**kw) for kw in (dict(n=4), dict(k=4), dict(q=True), dict(stats=True))]
    bad += [lambda: harness.KVLedger(model, None, new(whole, 1, 1, 2, 32), i32((1, 1, 2, 32)).to("meta"))]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    assert len(calls) == 6


@pytest.mark.parametrize("n", [0, 1, 7, 8, 9, 4096])
def test_host_numbers_of_every_kind(n, binding):  # noqa: F811
    want = [i * 7 - 3 for i in range(n)]
    for values in (want, tuple(want), np.array(want, np.int64), [np.int32(v) for v in want], [float(v) for v in want], np.array(want, np.float32)):
        got = binding.host_i32(values)
        assert list(got)[:n] == want and len(got) >= 1
