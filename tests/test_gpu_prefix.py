"""Attention of a batch behind a shared prefix (mn_prefix_attention) against the definition in 64 bits, every element within the
bound of attention_bounds.py, and a life of prompt, branches, steps and retirement through all the entry points together."""
import numpy as np
import pytest
import torch

from paper_2402_15678_amd import synth
from tests.attention_bounds import attend, check, factors, levels, ties

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "f32": torch.float32}


class Batch:
    """Sequences with own[b] tokens behind a prefix of P, ks[b] + 1 query rows each.  Slots that hold no token are not a number."""

    def __init__(self, H, Hkv, hd, kind, P, own, ks, seed, bs=16, spare=0, scale=1.0):
        from paper_2402_15678_amd import harness
        self.kind, self.P, self.ks, self.H, self.Hkv, self.hd, self.bs = kind, P, list(ks), H, Hkv, hd, bs
        self.ctx = [P + x for x in own]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        tot = [c + k + 1 for c, k in zip(self.ctx, ks)]
        p = P // bs
        need = [-(-t // bs) - p for t in tot]
        nb = p + sum(need) + spare
        ids = np.random.default_rng(seed).permutation(nb).astype(np.int32)
        self.table = np.full((len(ks), p + max(need)), -1, np.int32)
        self.table[:, :p] = ids[:p]
        at = p
        self.kp = torch.full((nb, Hkv, hd // 8, bs, 8), float("nan"), dtype=DT[kind], device="cuda")
        self.vp = torch.full((nb, Hkv, hd, bs), float("nan"), dtype=DT[kind], device="cuda")

        def fill(blk, n):
            self.kp[blk, :, :, :n] = torch.randn((Hkv, hd // 8, n, 8), generator=g, device="cuda").to(DT[kind])
            self.vp[blk, :, :, :n] = torch.randn((Hkv, hd, n), generator=g, device="cuda").to(DT[kind])
        for i in range(p):
            fill(int(ids[i]), bs)
        for b, m in enumerate(need):
            self.table[b, p:p + m] = ids[at:at + m]
            at += m
            for i in range(m):
                fill(int(self.table[b, p + i]), min(bs, tot[b] - (p + i) * bs))
        self.q = (torch.randn((sum(ks) + len(ks), H, hd), generator=g, device="cuda") * scale).to(DT[kind])
        self.d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if kind == "f16" else synth.DT_F32, 1, 128, H, Hkv, hd, 128, 8, 1 << 20)
        self.model = harness.DeviceModel.random_on_device(self.d, 1)
        self.max_ctx = max(tot)

    def kv(self):
        from paper_2402_15678_amd import harness
        return harness.DeviceKV(self.d, self.bs, self.kp.shape[0], self.table, self.ctx, [self.kp], [self.vp])

    def run(self, kv=None, spec=None, max_ctx=None, P=None):
        from paper_2402_15678_amd import harness
        ses = harness.PrefixSession(self.model, kv or self.kv(), len(self.ks), len(self.q), self.P if P is None else P, max_ctx or self.max_ctx)
        out = torch.full((len(self.q), self.H * self.hd), -7.0, dtype=DT[self.kind], device="cuda")
        ses.attention(self.q, torch.tensor(self.ks if spec is None else spec, dtype=torch.int32, device="cuda"), self.ks, out)
        torch.cuda.synchronize()
        return out, ses.dev_status.item()

    def rows(self, b):
        a = sum(self.ks[:b]) + b
        return slice(a, a + self.ks[b] + 1)

    def dense(self, b):
        n = self.ctx[b] + self.ks[b] + 1
        ids = torch.from_numpy(self.table[b, :-(-n // self.bs)].astype(np.int64)).cuda()
        return (self.kp[ids].permute(0, 3, 1, 2, 4).reshape(-1, self.Hkv, self.hd)[:n], self.vp[ids].permute(0, 3, 1, 2).reshape(-1, self.Hkv, self.hd)[:n])

    def check(self, out, seqs=None):
        for b in range(len(self.ks)) if seqs is None else seqs:
            r = self.rows(b)
            k, v = self.dense(b)
            check(out[r], *attend(self.q[r], k, v, torch.arange(self.ctx[b], self.ctx[b] + self.ks[b] + 1, device="cuda"), self.kind == "f16"))


GEOMETRIES = [(64, 8, 128, "f16"), (4, 4, 128, "f16"), (12, 12, 64, "f16"), (6, 2, 64, "f16"), (128, 2, 64, "f16"), (4, 4, 64, "f32"),
              (8, 2, 128, "f32"), (6, 2, 32, "f32"), (8, 8, 8, "f32"), (2, 2, 256, "f32"), (8, 8, 32, "f16"), (8, 2, 256, "f16")]


@pytest.mark.parametrize("H,Hkv,hd,kind", GEOMETRIES)
@pytest.mark.parametrize("P,own,ks", [(48, [0, 30, 7], [4, 0, 2]), (0, [0, 63, 64, 5], [0, 8, 1, 3]), (16, [0], [0]),
                                      (1040, [0, 1, 15, 16, 17, 200], [0, 0, 3, 0, 12, 1])], ids=str)
def test_prefix_matches_the_definition(H, Hkv, hd, kind, P, own, ks):
    x = Batch(H, Hkv, hd, kind, P, own, ks, H + hd + P)
    out, status = x.run()
    assert status == 0
    x.check(out)


@pytest.mark.parametrize("H,Hkv,hd,kind,P,own,ks", [
    (64, 8, 128, "f16", 4096, [300, 0, 900, 40, 16, 77, 5, 1500], [8] * 8), (64, 8, 128, "f16", 6000, [0, 3], [0, 1]),
    (40, 40, 128, "f16", 512, [9, 100, 2000], [0, 4, 1]), (8, 8, 128, "f16", 2048, [10] * 40, [0] * 40), (12, 12, 64, "f16", 1000 // 16 * 16, [33] * 12, [7] * 12),
    (4, 4, 64, "f32", 800, [100, 1, 40], [3, 0, 9]), (64, 8, 128, "f16", 128, [5, 700], [130, 0]), (8, 1, 64, "f16", 20000, [2500, 1], [0, 2])])
def test_long_prefixes_and_ragged_batches(H, Hkv, hd, kind, P, own, ks):
    x = Batch(H, Hkv, hd, kind, P, own, ks, 5)
    out, status = x.run()
    assert status == 0
    x.check(out)
    # sizes beyond the batch's own: a longer bound on the contexts
    again, status = x.run(max_ctx=min(x.table.shape[1] * x.bs, x.max_ctx + 11))
    assert status == 0
    x.check(again)


@pytest.mark.parametrize("H,Hkv,hd,kind,bs", [(4, 2, 128, "f16", 8), (6, 2, 32, "f32", 5), (12, 12, 64, "f16", 32), (8, 8, 8, "f32", 1)])
def test_other_block_sizes(H, Hkv, hd, kind, bs):
    x = Batch(H, Hkv, hd, kind, 3 * bs * 8, [0, 2 * bs + 1, 40], [3, 0, 5], 6, bs=bs)
    out, status = x.run()
    assert status == 0
    x.check(out)


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f32", 16)])
@pytest.mark.parametrize("count", [64, 65, 1100])
def test_many_sequences(kind, hd, count):
    g = np.random.default_rng(count)
    x = Batch(4, 2, hd, kind, 64, g.integers(0, 40, count).tolist(), g.integers(0, 4, count).tolist(), 7)
    out, status = x.run()
    assert status == 0
    x.check(out, sorted(set(g.integers(0, count, 40).tolist())))
    assert not (out == -7.0).all(dim=1).any()


def test_scores_far_apart_between_the_parts():
    """A row's weight is all in the prefix, all in its own keys, or in one key of either."""
    for kind, hd in (("f16", 128), ("f16", 64), ("f32", 64)):
        x = Batch(4, 2, hd, kind, 512, [100, 30], [3, 3], 8, scale=15.0)
        x.kp[:] = torch.where(torch.isnan(x.kp), x.kp, x.kp * 4)
        out, status = x.run()
        assert status == 0
        x.check(out)


def test_agrees_with_the_attention_that_reads_the_prefix_for_everybody():
    from paper_2402_15678_amd import binding, harness
    x = Batch(64, 8, 128, "f16", 1024, [50, 600, 0, 333], [8, 8, 8, 8], 9)
    out, _ = x.run()
    kv = x.kv()
    n = binding.mn_workspace_bytes(x.model.ctx, 4, len(x.q), x.max_ctx)
    ws, st = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    want = torch.zeros_like(out)
    binding.mn_attention(x.model.ctx, x.q.data_ptr(), torch.tensor(x.ks, dtype=torch.int32, device="cuda").data_ptr(), binding.host_i32(x.ks), 4,
                         x.max_ctx, kv.c, 0, want.data_ptr(), ws.data_ptr(), n, st.data_ptr(), harness.stream_ptr())
    torch.cuda.synchronize()
    # either is within its own bound of the definition; mn_attention rounds its scaled queries to fp16 as well
    for b in range(4):
        r = x.rows(b)
        k, v = x.dense(b)
        _, bound = attend(x.q[r], k, v, torch.arange(x.ctx[b], x.ctx[b] + 9, device="cuda"), True)
        assert ((out[r].double() - want[r].double()).abs() <= 2 * bound + 2e-2).all()


def test_damaged_sequences_get_zeros_and_the_others_their_results():
    from paper_2402_15678_amd import binding
    x = Batch(8, 2, 128, "f16", 128, [20, 40, 60, 5, 33, 17], [2, 0, 5, 1, 3, 4], 10, spare=2)
    good = x.table.copy()
    whole, status = x.run()
    assert status == 0
    cases = [("another prefix", lambda t, c: t.__setitem__((2, 3), (t[2, 3] + 1) % x.kp.shape[0]), 2, binding.MN_DEV_BLOCK_TABLE),
             ("a wild id", lambda t, c: t.__setitem__((4, 9), 1 << 30), 4, binding.MN_DEV_BLOCK_TABLE),
             ("a negative id", lambda t, c: t.__setitem__((5, 8), -1), 5, binding.MN_DEV_BLOCK_TABLE),
             ("a context inside the prefix", lambda t, c: c.__setitem__(1, 127), 1, binding.MN_DEV_CTX),
             ("a context beyond the bound", lambda t, c: c.__setitem__(3, x.max_ctx), 3, binding.MN_DEV_CTX)]
    for name, damage, b, flag in cases:
        ctx = list(x.ctx)
        x.table = good.copy()
        damage(x.table, x.ctx)
        out, status = x.run(kv=x.kv())
        x.table, x.ctx = good, ctx
        assert status == flag, name
        r = x.rows(b)
        assert (out[r] == 0).all(), name
        rest = torch.ones(len(out), dtype=torch.bool, device="cuda")
        rest[r] = False
        assert torch.equal(out[rest], whole[rest]), name
    # the first row is what is read: with an id out of range there, everybody differs from it or holds it
    x.table = good.copy()
    x.table[0, 2] = 1 << 30
    out, status = x.run(kv=x.kv())
    x.table = good
    assert status == binding.MN_DEV_BLOCK_TABLE and (out == 0).all()
    for spec in ([2, 0, 5, 1, 3, 5], [3, 0, 5, 1, 2, -1], [2, 0, 6, 0, 3, 4]):
        out, status = x.run(spec=spec)
        assert status == binding.MN_DEV_SPEC_LEN and (out == 0).all()


def test_pages_beyond_four_gigabytes():
    """Offsets into the pages pass 32 bits, in the attention and in the pool's copies."""
    from paper_2402_15678_amd import harness
    H, Hkv, hd, bs, nb = 16, 8, 128, 16, 140000
    x = Batch(H, Hkv, hd, "f16", 64, [20, 7], [1, 0], 11)
    far = {int(i): nb - 1 - int(i) * 7 for i in x.table[x.table >= 0].tolist()}
    kp = torch.empty((nb, Hkv, hd // 8, bs, 8), dtype=torch.float16, device="cuda")
    vp = torch.empty((nb, Hkv, hd, bs), dtype=torch.float16, device="cuda")
    want, _ = x.run()
    for a, b in far.items():
        kp[b], vp[b] = x.kp[a], x.vp[a]
    x.table = np.vectorize(lambda i: far.get(int(i), -1))(x.table).astype(np.int32)
    x.kp, x.vp = kp, vp
    kv = x.kv()
    out, status = x.run(kv=kv)
    assert status == 0 and torch.equal(out, want)
    # the last free blocks are the far ones: everything else is taken
    pool = harness.KVPool.from_tables(x.model, kv)
    pool.block_refs[:nb - 200] = 1
    assert pool.compact().item() > nb - 200
    out, status = x.run(kv=kv)
    assert status == 0 and torch.equal(out, want)


def test_same_numbers_on_another_stream_and_from_a_graph():
    from paper_2402_15678_amd import harness
    x = Batch(64, 8, 128, "f16", 2048, [50, 600, 0, 333], [8, 0, 8, 3], 12)
    want, _ = x.run()
    kv = x.kv()
    ses = harness.PrefixSession(x.model, kv, 4, len(x.q) + 9, 2048, x.max_ctx)
    spec, out = torch.tensor(x.ks, dtype=torch.int32, device="cuda"), torch.zeros_like(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ses.attention(x.q, spec, x.ks, out)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ses.attention(x.q, spec, x.ks, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and ses.dev_status.item() == 0
        assert torch.equal(x.run()[0], want)


@pytest.mark.parametrize("H,Hkv,hd,kind", [(16, 4, 128, "f16"), (4, 4, 64, "f32")])
def test_a_prompt_branches_steps_and_retires(H, Hkv, hd, kind):
    """One prompt enters the cache through the prompt attention, becomes four requests, each writes rows of its own (through the
    prompt attention's cache writes into a scratch table, copied in place), all attend behind the shared prompt, two leave, the pool is
    packed, and the rest attend again with the same results."""
    from paper_2402_15678_amd import harness
    bs, n, own, B = 16, 100, 6, 4
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if kind == "f16" else synth.DT_F32, 1, 128, H, Hkv, hd, 128, 8, 4096)
    model = harness.DeviceModel.random_on_device(d, 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    blocks = 40
    kp = torch.full((blocks, Hkv, hd // 8, bs, 8), float("nan"), dtype=DT[kind], device="cuda")
    vp = torch.full((blocks, Hkv, hd, bs), float("nan"), dtype=DT[kind], device="cuda")
    kv = harness.DeviceKV(d, bs, blocks, np.full((B, 10), -1, np.int32), [0] * B, [kp], [vp])
    pool = harness.KVPool.from_tables(model, kv)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    pool.reserve(dev([n]))
    rows = torch.randn((n, H + 2 * Hkv, hd), generator=g, device="cuda").to(DT[kind])
    q, k, v = rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:]
    out = torch.zeros((n, H * hd), dtype=DT[kind], device="cuda")
    harness.prompt_attention(model, q, k, v, dev([0, n]), harness.PromptRows([0, n]), out, kv, 0, pool.dev_status)
    check(out, *attend(q, k, v, torch.arange(n, device="cuda"), kind == "f16"))
    kv.ctx_lens[:1] = n
    pool.fork(dev([0, 0, 0]), dev([1, 2, 3]))
    pool.reserve(dev([n + own] * B))
    torch.cuda.synchronize()
    assert pool.dev_status.item() == 0 and pool.seq_blocks.tolist() == [7] * B
    table = kv.block_tables.cpu().numpy()
    new = torch.randn((B, own, H + 2 * Hkv, hd), generator=g, device="cuda").to(DT[kind])
    for b in range(B):
        for i in range(own):
            blk, off = int(table[b, (n + i) // bs]), (n + i) % bs
            kp[blk, :, :, off] = new[b, i, H:H + Hkv].reshape(Hkv, -1, 8)
            vp[blk, :, :, off] = new[b, i, H + Hkv:]
    P = n // bs * bs
    ses = harness.PrefixSession(model, kv, B, B * own, P, n + own)
    got = ses.attention(new[:, :, :H].reshape(B * own, H, hd).contiguous(), dev([own - 1] * B), [own - 1] * B,
                        torch.zeros((B * own, H * hd), dtype=DT[kind], device="cuda"))
    for b in range(B):
        check(got[b * own:(b + 1) * own], *attend(new[b, :, :H], torch.cat((k, new[b, :, H:H + Hkv])), torch.cat((v, new[b, :, H + Hkv:])),
                                                  torch.arange(n, n + own, device="cuda"), kind == "f16"))
    pool.free(dev([0, 2]))
    live = pool.compact()
    assert live.item() == 6 + 2
    order = dev([1, 3])
    packed = harness.DeviceKV(d, bs, blocks, kv.block_tables[order.long()].cpu().numpy(), [n, n], [kp], [vp])
    ses2 = harness.PrefixSession(model, packed, 2, 2 * own, P, n + own)
    again = ses2.attention(new[[1, 3], :, :H].reshape(2 * own, H, hd).contiguous(), dev([own - 1] * 2), [own - 1] * 2,
                           torch.zeros((2 * own, H * hd), dtype=DT[kind], device="cuda"))
    torch.cuda.synchronize()
    assert ses.dev_status.item() == 0 and ses2.dev_status.item() == 0 and pool.dev_status.item() == 0
    for i, b in enumerate((1, 3)):
        assert torch.equal(again[i * own:(i + 1) * own], got[b * own:(b + 1) * own])


def _same(got, want):
    """Bit for bit, NaN where there is NaN."""
    off = ~((got == want) | (got.isnan() & want.isnan()))
    assert not off.any().item(), f"{int(off.sum())} elements, the first (row, head, element) {off.nonzero()[0].tolist()}: {got[off][0].item()}, not {want[off][0].item()}"


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (4, 4, 128, "f16"), (12, 12, 64, "f16"), (4, 4, 64, "f32"), (8, 2, 128, "f32"), (8, 8, 8, "f32"),
                                           (2, 2, 256, "f32"), (8, 2, 256, "f16")])
@pytest.mark.parametrize("at", [0, 2, 20])
def test_what_is_not_finite_reaches_the_rows_that_see_it(H, Hkv, hd, kind, at):
    """Infinities and NaN in the values of one scored token of one sequence: the rows before it, other elements, other KV heads and other
    sequences keep their bits."""
    x = Batch(H, Hkv, hd, kind, 64, [37, 5, 0], [2, 24, 4], 18)
    plain, status = x.run()
    assert status == 0
    odd = {1: float("inf"), 3: float("-inf"), 6: float("nan"), hd - 1: float("inf")}
    pos = x.ctx[1] + at
    for e, y in odd.items():
        x.vp[int(x.table[1, pos // x.bs]), Hkv - 1, e, pos % x.bs] = y
    out, status = x.run()
    assert status == 0
    want = plain.clone().view(-1, H, hd)
    r = x.rows(1)
    for e, y in odd.items():
        want[r.start + at:r.stop, (Hkv - 1) * (H // Hkv):, e] = y
    _same(out.view_as(want), want)


@pytest.mark.parametrize("kind,hd,bs", [("f16", 128, 16), ("f16", 64, 16), ("f32", 32, 8)])
@pytest.mark.parametrize("count", [5, 64, 65, 1030])
def test_emptied_slots_in_a_batch(kind, hd, bs, count):
    """Slots without tokens and blocks get zeros, the first ones among them, and nobody else notices."""
    from paper_2402_15678_amd import binding
    g = np.random.default_rng(count)
    x = Batch(4, 2, hd, kind, 4 * bs, g.integers(0, 50, count).tolist(), g.integers(0, 4, count).tolist(), count, bs=bs)
    whole, status = x.run()
    assert status == 0
    gone = [0, 1, count - 1]
    for b in gone:
        x.table[b] = -1
        x.ctx[b] = 0
    out, status = x.run(kv=x.kv())
    assert status == binding.MN_DEV_CTX
    rest = torch.ones(len(out), dtype=torch.bool, device="cuda")
    for b in gone:
        assert (out[x.rows(b)] == 0).all()
        rest[x.rows(b)] = False
    assert torch.equal(out[rest], whole[rest])
    # nobody left
    x.table[:] = -1
    x.ctx = [0] * count
    out, status = x.run(kv=x.kv())
    assert status == binding.MN_DEV_CTX and (out == 0).all()


@pytest.mark.parametrize("count", [6, 70])
def test_two_batches_on_two_streams_at_once(count):
    """Workspaces of their own: neither call sees the other, eager or replayed, step after step."""
    from paper_2402_15678_amd import harness
    xs = [Batch(16, 4, 128, "f16", 512, [30 + i] * count, [2] * count, 20 + i) for i in range(2)]
    want = [x.run()[0] for x in xs]
    sets = []
    for x in xs:
        kv = x.kv()
        ses = harness.PrefixSession(x.model, kv, count, len(x.q), x.P, x.max_ctx)
        spec = torch.tensor(x.ks, dtype=torch.int32, device="cuda")
        out = torch.full((len(x.q), x.H * x.hd), -7.0, dtype=torch.float16, device="cuda")
        sets.append((ses, spec, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, (ses, spec, out, st) in zip(xs, sets):
            with torch.cuda.stream(st):
                ses.attention(x.q, spec, x.ks, out)
    torch.cuda.synchronize()
    for w, (ses, spec, out, st) in zip(want, sets):
        assert torch.equal(out, w) and ses.dev_status.item() == 0
    graphs = []
    for x, (ses, spec, out, st) in zip(xs, sets):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            ses.attention(x.q, spec, x.ks, out)
        graphs.append(gr)
    for _ in range(5):
        for s in sets:
            s[2].zero_()
        torch.cuda.synchronize()
        for gr, (ses, spec, out, st) in zip(graphs, sets):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for w, s in zip(want, sets):
            assert torch.equal(s[2], w)


def test_damaged_sequences_in_a_large_batch():
    """More than 64 sequences (a work list): who fails gets zeros, the others their results; lengths that do not add up, everybody."""
    from paper_2402_15678_amd import binding
    count = 90
    g = np.random.default_rng(3)
    x = Batch(8, 2, 128, "f16", 64, g.integers(0, 90, count).tolist(), g.integers(0, 5, count).tolist(), 31, spare=1)
    good, ctx = x.table.copy(), list(x.ctx)
    whole, status = x.run()
    assert status == 0
    damages = [(lambda: x.table.__setitem__((66, 1), (x.table[66, 1] + 1) % x.kp.shape[0]), [66], binding.MN_DEV_BLOCK_TABLE),
               (lambda: x.table.__setitem__((89, x.ctx[89] // 16), 1 << 30), [89], binding.MN_DEV_BLOCK_TABLE),
               (lambda: (x.ctx.__setitem__(3, 63), x.ctx.__setitem__(70, 0)), [3, 70], binding.MN_DEV_CTX),
               (lambda: x.ctx.__setitem__(80, 1 << 30), [80], binding.MN_DEV_CTX),
               (lambda: x.ctx.__setitem__(0, -5), [0], binding.MN_DEV_CTX)]
    for damage, gone, flag in damages:
        damage()
        out, status = x.run(kv=x.kv(), max_ctx=max(ctx) + 6)
        x.table, x.ctx = good.copy(), list(ctx)
        assert status == flag
        rest = torch.ones(len(out), dtype=torch.bool, device="cuda")
        for b in gone:
            assert (out[x.rows(b)] == 0).all()
            rest[x.rows(b)] = False
        x.check(out, [b for b in (1, 2, 65, 67, 88) if b not in gone])
        assert torch.equal(out[rest], x.run(max_ctx=max(ctx) + 6)[0][rest])
    for at, by in ((5, 1), (89, -9), (70, 40)):
        spec = list(x.ks)
        spec[at] += by
        out, status = x.run(spec=spec)
        assert status == binding.MN_DEV_SPEC_LEN and (out == 0).all()


@pytest.mark.parametrize("kind,hd,P", [("f16", 128, 1024), ("f16", 64, 512), ("f32", 64, 256), ("f16", 256, 128)])
@pytest.mark.parametrize("far", [True, False], ids=["far", "mixed"])
def test_prefix_scores_at_the_end_of_the_range(kind, hd, P, far):
    x = Batch(4, 2, hd, kind, P, [100, 0, 600], [3, 2, 8], 21)
    nb = len(x.kp)
    level = levels(nb * x.bs, "any", 5).view(nb, 1, 1, x.bs, 1)
    x.kp[:] = torch.where(x.kp.isnan(), x.kp, (level * (8188.0 if kind == "f16" else 2.0 ** 50)).to(x.kp.dtype).expand_as(x.kp))
    f = torch.full((len(x.q),), 65504.0 if kind == "f16" else 2.0 ** 53, device="cuda") if far else factors(len(x.q), kind, 6)
    x.q[:] = f.view(-1, 1, 1).to(x.q.dtype)
    out, status = x.run()
    assert status == 0
    for b in range(3):
        r, (k, v) = x.rows(b), x.dense(b)
        want, bound = ties(x.q[r], k, v, torch.arange(x.ctx[b], x.ctx[b] + x.ks[b] + 1, device="cuda"))
        check(out[r], want, bound + (2.0 ** -11 if kind == "f16" else 2.0 ** -24) * want.abs() + (2.0 ** -25 if kind == "f16" else 0))


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (12, 12, 64, "f16"), (4, 4, 64, "f32"), (8, 2, 256, "f16")])
@pytest.mark.parametrize("count", [3, 70])
def test_prefix_row_whose_scores_are_all_minus_infinity(H, Hkv, hd, kind, count):
    x = Batch(H, Hkv, hd, kind, 64, [37, 5, 0] + [1] * (count - 3), [2, 24, 4] + [0] * (count - 3), 24)
    x.kp[:, :, 0, :, 0] = -x.kp[:, :, 0, :, 0].abs() - 1
    plain, status = x.run()
    assert status == 0
    at = x.rows(1).start + 9
    x.q[at, H - 1, 0] = float("inf")
    out, status = x.run()
    assert status == 0
    want = plain.clone().view(-1, H, hd)
    want[at, H - 1] = float("nan")
    _same(out.view_as(want), want)


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (8, 8, 8, "f32"), (16, 4, 8, "f16"), (8, 2, 256, "f16")])
@pytest.mark.parametrize("at", [5, 70])
def test_prefix_key_at_minus_infinity_has_no_weight(H, Hkv, hd, kind, at):
    """One of the shared keys, or one of a sequence's own, at minus infinity."""
    e = hd - 3
    x = Batch(H, Hkv, hd, kind, 64, [37, 15], [2, 4], 26)
    x.kp[int(x.table[0, at // x.bs]), :, e // 8, at % x.bs, e % 8] = float("inf")
    out, status = x.run()
    assert status == 0
    for b in range(2):
        r, (k, v) = x.rows(b), x.dense(b)
        limit = torch.arange(x.ctx[b], x.ctx[b] + x.ks[b] + 1, device="cuda")
        hit = at < x.P or b == 0
        rest = torch.arange(len(k), device="cuda") != (at if hit else -1)
        want, bound = attend(x.q[r], k[rest], v[rest], limit - int(hit), kind == "f16")
        up = (hit & (x.q[r][:, :, e] > 0))[:, :, None].expand(-1, H, hd).reshape(len(want), -1)
        assert out[r][up].isnan().all()
        check(torch.where(up, want.to(out.dtype), out[r]), want, bound + 2.0 ** -11 * want.abs() + 2.0 ** -25)


def test_agrees_with_the_attention_that_reads_the_prefix_for_everybody_within_the_roundings():
    """Either is within its bound of the definition at the queries that it multiplies: mn_attention rounds them to fp16 once scaled.  What is left
    shows a mask that is off by one key."""
    from paper_2402_15678_amd import binding, harness
    x = Batch(64, 8, 128, "f16", 1024, [50, 600, 0, 333], [8, 8, 8, 8], 9)
    out, _ = x.run()
    kv = x.kv()
    n = binding.mn_workspace_bytes(x.model.ctx, 4, len(x.q), x.max_ctx)
    ws, st = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    other = torch.zeros_like(out)
    binding.mn_attention(x.model.ctx, x.q.data_ptr(), torch.tensor(x.ks, dtype=torch.int32, device="cuda").data_ptr(), binding.host_i32(x.ks), 4,
                         x.max_ctx, kv.c, 0, other.data_ptr(), ws.data_ptr(), n, st.data_ptr(), harness.stream_ptr())
    torch.cuda.synchronize()
    scale = 1.4426950408889634 / 128 ** 0.5
    rounded = (x.q.float() * scale).half().double() / scale
    for b in range(4):
        r = x.rows(b)
        k, v = x.dense(b)
        limit = torch.arange(x.ctx[b], x.ctx[b] + 9, device="cuda")
        want, bound = attend(x.q[r], k, v, limit, True)
        want2, bound2 = attend(rounded[r], k, v, limit, True)
        check(other[r], want2, bound2)
        slack = bound + bound2 + (want - want2).abs()
        assert ((out[r].double() - other[r].double()).abs() <= slack).all()
        shifted, _ = attend(x.q[r], k, v, limit - 1, True)
        assert ((shifted - other[r].double()).abs() > slack).any()
