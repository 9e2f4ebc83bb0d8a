"""The page pool (mn_kv_reserve, mn_kv_fork, mn_kv_free, mn_kv_compact) against its sequential definition: tables, references,
contexts and every page, all whole numbers or copies, so everything is compared exactly."""
import numpy as np
import pytest
import torch

from oracle import minions_oracle as orc
from paper_2402_15678_amd import synth

pytestmark = pytest.mark.gpu


def _setup(desc, bs, blocks, width, ctx, seed, damage=None):
    """Slots with `ctx` tokens each (0: empty), blocks scattered; the device pool and its definition side by side."""
    from paper_2402_15678_amd import harness
    g = synth.stream(91, seed)
    need = [-(-c // bs) for c in ctx]
    ids = g.permutation(blocks)
    table = np.full((len(ctx), width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    refs = np.zeros(blocks, np.int32)
    refs[ids[:at]] = 1
    held, ctx = np.array(need, np.int32), np.array(ctx, np.int32)
    if damage:
        damage(table, refs, held, ctx)
    dt = np.float16 if desc.dtype == synth.DT_BF16 else np.float32
    hk, hd, L = desc.n_kv_heads, desc.head_dim, desc.n_layers
    k = g.standard_normal((L, blocks, hk, hd // 8, bs, 8), dtype=np.float32).astype(dt)
    v = g.standard_normal((L, blocks, hk, hd, bs), dtype=np.float32).astype(dt)
    model = harness.DeviceModel.random_on_device(desc, 1)
    kv = harness.DeviceKV(desc, bs, blocks, table, ctx, [torch.from_numpy(a).cuda() for a in k], [torch.from_numpy(a).cuda() for a in v])
    pool = harness.KVPool(model, kv, torch.from_numpy(refs).cuda(), torch.from_numpy(held).cuda())
    want = orc.PagePool(table, refs, held, ctx, bs, [*k, *v])
    return pool, want


def _dev(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda:0")


def _compare(pool, want):
    torch.cuda.synchronize()
    assert np.array_equal(pool.kv.block_tables.cpu().numpy(), want.table)
    assert np.array_equal(pool.block_refs.cpu().numpy(), want.refs)
    assert np.array_equal(pool.seq_blocks.cpu().numpy(), want.held)
    assert np.array_equal(pool.kv.ctx_lens.cpu().numpy(), want.ctx)
    assert pool.dev_status.item() == want.status
    for t, p in zip([*pool.kv.k_pages, *pool.kv.v_pages], want.pages):
        assert np.array_equal(t.cpu().numpy(), p)


def _desc(layers=2, heads=2, hd=32, dtype=synth.DT_F32):
    return synth.ModelDesc(synth.ARCH_LLAMA, dtype, layers, 128, heads, heads, hd, 128, 8, 1 << 16)


DESCS = {"fp32": _desc(), "fp16": _desc(3, 4, 64, synth.DT_BF16), "layers": _desc(100, 2, 64, synth.DT_BF16), "narrow": _desc(1, 8, 8)}


@pytest.mark.parametrize("name,bs,blocks,seed", [("fp32", 16, 60, 1), ("fp16", 16, 130, 2), ("layers", 16, 40, 3), ("narrow", 5, 64, 4),
                                                 ("fp32", 1, 200, 5), ("fp16", 16, 3000, 6)])
def test_random_life_of_a_pool(name, bs, blocks, seed):
    """Requests come, branch, grow, commit and leave in random order, and the pool is packed now and then."""
    g = synth.stream(92, seed)
    slots, width = 12, max(4, min(20, blocks // 4))
    pool, want = _setup(DESCS[name], bs, blocks, width, [0, 3 * bs, 1, 2 * bs + 1] + [0] * (slots - 4), seed)
    for step in range(40):
        op = int(g.integers(0, 4))
        if op == 0:
            n = int(g.integers(1, 5))
            src, dst = g.integers(0, slots, n), g.integers(0, slots, n)
            pool.fork(_dev(src), _dev(dst))
            want.fork(src.tolist(), dst.tolist())
        elif op == 1:
            n = int(g.integers(1, slots + 1))
            tokens = want.ctx[:n] + g.integers(-2, 3 * bs, n)
            pool.reserve(_dev(tokens))
            want.reserve(tokens.tolist())
            # the step commits some of what there is room for; a cache may also be cut back
            commit = np.minimum(want.ctx + g.integers(-bs, 2 * bs, slots), want.held * bs).clip(0)
            want.ctx[:] = commit
            pool.kv.ctx_lens.copy_(_dev(commit))
        elif op == 2:
            gone = g.integers(0, slots, int(g.integers(1, 4)))
            pool.free(_dev(gone))
            want.free(gone.tolist())
        else:
            n = want.compact()
            assert pool.compact().item() == n
            assert (want.refs[:n] > 0).all() and (want.refs[n:] == 0).all()
        _compare(pool, want)
    assert (want.refs >= 0).all()


def test_children_write_into_pages_of_their_own():
    """A prompt of 2 and a half blocks in five branches: the whole blocks stay shared, the half one is copied for everybody that
    writes, and the original is free again once nobody holds it."""
    pool, want = _setup(DESCS["fp16"], 16, 30, 6, [40, 0, 0, 0, 0], 7)
    pool.fork(_dev([0, 0, 0, 0]), _dev([1, 2, 3, 4]))
    want.fork([0, 0, 0, 0], [1, 2, 3, 4])
    _compare(pool, want)
    assert sorted(want.refs.tolist())[-3:] == [5, 5, 5]
    for _ in range(2):                     # (the second call finds everything in place)
        pool.reserve(_dev([49] * 5))
        want.reserve([49] * 5)
        _compare(pool, want)
    rows = pool.kv.block_tables.cpu().numpy()
    assert (rows[:, :2] == rows[0, :2]).all() and len(set(rows[:, 2].tolist())) == 5 and len(set(rows[:, 3].tolist())) == 5


def test_many_slots_and_blocks():
    """4096 slots, 70000 blocks, more than one round of every loop in the plan."""
    d = _desc(1, 2, 32)
    g = synth.stream(93, 1)
    ctx = g.integers(0, 200, 4096).tolist()
    pool, want = _setup(d, 16, 70000, 20, ctx, 8)
    tokens = [c + int(x) for c, x in zip(ctx, g.integers(0, 60, 4096))]
    pool.reserve(_dev(tokens))
    want.reserve(tokens)
    _compare(pool, want)
    gone = g.permutation(4096)[:2000]
    pool.free(_dev(gone))
    want.free(gone.tolist())
    src = [s for s in range(4096) if want.held[s]][:1000]
    dst = [s for s in range(4096) if not want.held[s] and not want.ctx[s]][:1000]
    pool.fork(_dev(src), _dev(dst))
    want.fork(src, dst)
    _compare(pool, want)
    assert pool.compact().item() == want.compact()
    _compare(pool, want)


def test_what_a_pool_cannot_do_it_leaves_and_reports():
    from paper_2402_15678_amd import binding

    def damage(table, refs, held, ctx):
        table[2, 0] = 1 << 20            # a wild id
        held[3] = 0                      # a context without blocks
        held[4] = 99                     # more blocks than the row has
        ctx[5] = -3
        refs[table[6, 0]] = 0            # a block that counts as free although a row holds it
    pool, want = _setup(DESCS["fp32"], 16, 24, 5, [20, 0, 20, 20, 20, 20, 20, 0], 9, damage)
    for call, args in [("fork", ([2, 3, 5, 0], [1, 1, 7, 7])), ("fork", ([0, 0, 9, -1, 0], [0, 8, 1, 1, 2])), ("fork", ([0, 1], [1, 7])),
                       ("fork", ([5], [7])), ("reserve", ([30, 33, 30, 30, 30, 30, 20, 16 * 5 + 1],)), ("free", ([2, 2, 4, 6, -1, 8],)),
                       ("reserve", ([81, 81, 200, 0, -7, 5, 300, 300],)), ("reserve", ([80] * 8,)), ("free", ([0, 1, 2, 3, 4, 5, 6, 7],))]:
        want.status = 0
        pool.dev_status.zero_()
        getattr(pool, call)(*[_dev(a) for a in args])
        getattr(want, call)(*args)
        _compare(pool, want)
    assert binding.MN_DEV_POOL == want.EMPTY and binding.MN_DEV_SEQ == want.SLOT and binding.MN_DEV_BLOCK_TABLE == want.TABLE


def test_pool_exhaustion_serves_the_first_slots():
    pool, want = _setup(DESCS["fp16"], 16, 10, 8, [16, 16, 16, 16], 10)
    pool.reserve(_dev([48, 64, 33, 17]))   # 2, then 3, of 6 blocks; the third needs 2 and gets none, nor does the fourth
    want.reserve([48, 64, 33, 17])
    _compare(pool, want)
    assert want.status == want.EMPTY and want.held.tolist() == [3, 4, 1, 1]


def test_captured_pool_calls_replay():
    """Branch and retire in one graph, replayed on the mapping put back by a copy, against the eager calls."""
    pool, want = _setup(DESCS["fp16"], 16, 40, 6, [40, 23, 0, 0, 0], 11)
    saved = pool.state.clone()
    src, dst, tokens, gone = _dev([0, 0, 1]), _dev([2, 3, 4]), _dev([45, 30, 45, 60, 24]), _dev([0, 3])

    def life():
        pool.state.copy_(saved)
        pool.fork(src, dst)
        pool.reserve(tokens)
        pool.free(gone)
        pool.compact()

    want.fork([0, 0, 1], [2, 3, 4])
    want.reserve([45, 30, 45, 60, 24])
    want.free([0, 3])
    n = want.compact()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        life()
    torch.cuda.current_stream().wait_stream(stream)
    _compare(pool, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        life()
    for _ in range(3):
        pool.n_live.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert pool.n_live.item() == n
        assert np.array_equal(pool.kv.block_tables.cpu().numpy(), want.table)
        assert np.array_equal(pool.block_refs.cpu().numpy(), want.refs)
        life()
        torch.cuda.synchronize()
        assert np.array_equal(pool.kv.block_tables.cpu().numpy(), want.table)


@pytest.mark.parametrize("name", ["fp32", "fp16"])
def test_a_context_without_layers_has_the_pages_of_layer_0(name):
    """A context without layers, whose attention calls read layer 0's pages: these move with the blocks, and the table with them."""
    from paper_2402_15678_amd import harness
    pool, want = _setup(_desc(1, 2, 64, DESCS[name].dtype), 16, 30, 6, [40, 23, 0, 0, 50], 12)
    pool.model = harness.DeviceModel.random_on_device(pool.model.desc.with_layers(0), 1)
    for call, args in [("fork", ([0, 0], [2, 3])), ("reserve", ([45, 30, 45, 60, 51],)), ("free", ([0, 3],)), ("compact", ()), ("reserve", ([64] * 5,))]:
        got = getattr(pool, call)(*[_dev(a) for a in args])
        n = getattr(want, call)(*args)
        assert call != "compact" or got.item() == n
        _compare(pool, want)


def test_replayed_pool_calls_move_the_pages():
    """Branch, grow, retire and pack in one graph: before every replay mapping and pages are put back, after it all of it is compared."""
    pool, want = _setup(DESCS["fp16"], 16, 40, 6, [40, 23, 0, 0, 0], 13)
    pages = [*pool.kv.k_pages, *pool.kv.v_pages]
    saved, bytes_ = pool.state.clone(), [p.clone() for p in pages]
    src, dst, tokens, gone = _dev([0, 0, 1]), _dev([2, 3, 4]), _dev([45, 30, 45, 60, 24]), _dev([0, 3])

    def back():
        pool.state.copy_(saved)
        for p, b in zip(pages, bytes_):
            p.copy_(b)

    def life():
        pool.fork(src, dst)
        pool.reserve(tokens)
        pool.free(gone)
        pool.compact()

    want.fork([0, 0, 1], [2, 3, 4])
    want.reserve([45, 30, 45, 60, 24])
    want.free([0, 3])
    n = want.compact()
    assert any(not np.array_equal(a, b.cpu().numpy()) for a, b in zip(want.pages, bytes_))
    life()
    _compare(pool, want)
    back()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        life()
    for _ in range(3):
        back()
        pool.n_live.zero_()
        graph.replay()
        _compare(pool, want)
        assert pool.n_live.item() == n
        back()
        life()
        _compare(pool, want)


def test_fork_and_free_need_no_context():
    from paper_2402_15678_amd import binding, harness
    pool, want = _setup(DESCS["fp32"], 16, 24, 5, [20, 33, 0, 0], 14)
    src, dst, gone = _dev([0, 1]), _dev([3, 2]), _dev([1, 3])
    binding.mn_kv_fork(None, pool.kv.c, pool.c, src.data_ptr(), dst.data_ptr(), 2, pool.dev_status.data_ptr(), harness.stream_ptr())
    binding.mn_kv_free(None, pool.kv.c, pool.c, gone.data_ptr(), 2, pool.dev_status.data_ptr(), harness.stream_ptr())
    want.fork([0, 1], [3, 2])
    want.free([1, 3])
    _compare(pool, want)
