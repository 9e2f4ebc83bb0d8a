"""The weight that attention gives to every cached token (mn_kv_weigh), the eviction that goes by it (mn_kv_evict), and a life of prompt,
steps and evictions through all the entry points of a bounded cache together."""
import math

import numpy as np
import pytest
import torch

from paper_2402_15678_amd import synth
from tests.attention_bounds import attend, check
from tests.test_gpu_window import Batch

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "f32": torch.float32}
LOG2E = 1.4426950408889634
GEOMETRIES = [(64, 8, 128, "f16"), (4, 4, 128, "f16"), (12, 12, 64, "f16"), (6, 2, 64, "f16"), (128, 2, 64, "f16"), (4, 4, 64, "f32"), (8, 2, 128, "f32"),
              (6, 2, 32, "f32"), (8, 8, 8, "f32"), (2, 2, 256, "f32"), (8, 8, 32, "f16"), (8, 2, 256, "f16"), (8, 2, 16, "f32")]


class Weighed(Batch):
    """A Batch with statistics, worked out here, and a ledger with something in it."""

    def __init__(self, H, Hkv, hd, kind, ctx, ks, seed, bs=16, extra=0, slots=0):
        from paper_2402_15678_amd import harness
        super().__init__(H, Hkv, hd, kind, ctx, ks, 1 << 20, 0, seed, bs=bs, blind=False, spare=2)
        self.stats = torch.zeros((len(self.q), H, 2), device="cuda")
        for b in range(len(ks)):
            for h in range(H):
                s = self.scores(b, h) * LOG2E
                m = s.amax(dim=1).float() + (h % 3 - 1) * 2.5       # (a reference, not the maximum)
                self.stats[self.rows(b), h, 0] = m
                self.stats[self.rows(b), h, 1] = torch.exp2(s - m.double()[:, None]).sum(dim=1).float()
        self.width, self.slots = self.max_ctx + extra, len(ks) + slots
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        shape = (1, self.slots, Hkv, self.width)
        self.mass0 = torch.rand(shape, generator=g, device="cuda") * 5
        self.born0 = torch.full(shape, -5, dtype=torch.int32, device="cuda")
        self.ledger = harness.KVLedger(self.model, self.kv(), self.mass0.clone(), self.born0.clone())

    def scores(self, b, h):
        k, _ = self.dense(b)
        s = self.q[self.rows(b)][:, h].double() @ k[:, h // (self.H // self.Hkv)].double().t().contiguous() / math.sqrt(self.hd)
        return s.masked_fill(~self.visible(b), -math.inf)

    def weigh(self, kv=None, n_out=None, seen=None, spec=None, max_ctx=None):
        dev = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.ledger.kv = kv or self.kv()
        self.ledger.mass.copy_(self.mass0)
        self.ledger.born.copy_(self.born0)
        self.ledger.dev_status.zero_()
        self.ledger.weigh(self.q, self.stats, dev(self.ks if spec is None else spec), self.ks, 0, max_ctx or self.max_ctx, dev(n_out), dev(seen))
        torch.cuda.synchronize()
        return self.ledger.dev_status.item()

    def check_weights(self, counts=None, seen=None, seqs=None, lost=()):
        """counts[b] rows of each sequence.  Off by: the scores' error and the reference's rounding, as relative errors of a weight
        (times ln 2, of the exponent), 2^-21 of exponential and quotient, and an addition's 2^-24 per row."""
        G = self.H // self.Hkv
        counts = counts or [k + 1 for k in self.ks]
        mass, born = self.mass0.double(), self.born0.clone()
        bound = torch.zeros_like(mass)
        for b in range(len(self.ks)) if seqs is None else seqs:
            c, n = self.ctx[b], counts[b]
            if n <= 0:
                continue
            k, _ = self.dense(b)
            for g in range(self.Hkv):
                total, err = torch.zeros(c + n, dtype=torch.float64, device="cuda"), 0
                for h in range(g * G, (g + 1) * G):
                    st = self.stats[self.rows(b), h].double()[:n]
                    p = torch.exp2(self.scores(b, h)[:n, :c + n] * LOG2E - st[:, :1]) / st[:, 1:]
                    total += p.sum(dim=0)
                    q = self.q[self.rows(b)][:n, h].double().abs()
                    mag = (q @ k[:, g].double().abs().t().contiguous() / math.sqrt(self.hd)).amax()
                    err = max(err, float(2 * (self.hd * 2.0 ** -24 * mag + 2.0 ** -22 * mag) + 2.0 ** -23 * st[:, 0].abs().amax() + 2.0 ** -21))
                old = mass[0, b, g, :c].clone()
                mass[0, b, g, :c] += total[:c]
                mass[0, b, g, c:c + n] = total[c:]
                bound[0, b, g, :c + n] = total * (err + (n * G + 8) * 2.0 ** -24) + 1e-30
                bound[0, b, g, :c] += (old + total[:c]) * 2.0 ** -24
                born[0, b, g, c:c + n] = (c if seen is None else seen[b]) + torch.arange(n, device="cuda", dtype=torch.int32)
        for b, slots in lost:
            mass[0, b, :, slots], bound[0, b, :, slots], born[0, b, :, slots] = self.mass0[0, b, :, slots].double(), 0, self.born0[0, b, :, slots]
        over = (self.ledger.mass.double() - mass).abs() - bound
        assert over.max() <= 0, (over.max(), (over > 0).nonzero()[:5])
        assert torch.equal(self.ledger.born, born)


@pytest.mark.parametrize("H,Hkv,hd,kind", GEOMETRIES)
@pytest.mark.parametrize("ctx,ks", [([0, 30, 7], [4, 0, 2]), ([0, 63, 64, 5, 300], [0, 8, 1, 3, 40]), ([0], [150])], ids=str)
def test_weights_match_the_definition(H, Hkv, hd, kind, ctx, ks):
    x = Weighed(H, Hkv, hd, kind, ctx, ks, H + hd, extra=3, slots=2)
    assert x.weigh() == 0
    x.check_weights()
    assert x.weigh(seen=[c + 1000 * b for b, c in enumerate(ctx)], max_ctx=min(x.width, x.table.shape[1] * 16)) == 0
    x.check_weights(seen=[c + 1000 * b for b, c in enumerate(ctx)])


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (12, 12, 64, "f16"), (4, 4, 64, "f32"), (8, 2, 256, "f16")])
def test_weights_behind_the_commit(H, Hkv, hd, kind):
    """The accepted rows are the end of the context; the others leave no trace."""
    from paper_2402_15678_amd import harness
    x = Weighed(H, Hkv, hd, kind, [50, 0, 333, 17], [8, 3, 8, 0], 3)
    for n in ([9, 4, 9, 1], [1, 2, 5, 1], [3, 0, -1, 1]):
        ctx = [c + max(a, 0) for c, a in zip(x.ctx, n)]
        kv = harness.DeviceKV(x.d, x.bs, x.kp.shape[0], x.table, ctx, [x.kp], [x.vp])
        assert x.weigh(kv=kv, n_out=n) == 0
        x.check_weights(n)


@pytest.mark.parametrize("hd,kind,bs", [(128, "f16", 8), (32, "f32", 5), (64, "f16", 32), (8, "f32", 1)])
def test_weights_of_other_block_sizes(hd, kind, bs):
    x = Weighed(max(4, 64 // hd), 2, hd, kind, [0, 2 * bs + 1, 150], [3, 0, 5], 4, bs=bs)
    assert x.weigh() == 0
    x.check_weights()


@pytest.mark.parametrize("count", [64, 300])
def test_weights_of_many_sequences(count):
    g = np.random.default_rng(count)
    x = Weighed(2, 1, 64, "f16", g.integers(0, 60, count).tolist(), g.integers(0, 4, count).tolist(), 5)
    assert x.weigh() == 0
    x.check_weights()


def test_long_contexts_and_prompts():
    for H, Hkv, hd, kind, ctx, ks in ((16, 2, 128, "f16", [9000], [8]), (4, 2, 128, "f16", [0, 300], [1500, 700]), (2, 2, 64, "f32", [0], [900]),
                                      (6, 2, 128, "f16", [40, 0], [350, 1]), (40, 40, 128, "f16", [700] * 8, [200] * 8), (12, 12, 64, "f16", [700, 3] * 8, [100, 230] * 8),
                                      (16, 2, 64, "f16", [0], [5000]), (40, 40, 128, "f16", [900, 11] * 4, [120, 150] * 4), (8, 8, 64, "f16", [0], [1100]),
                                      (8, 8, 64, "f16", [9000] * 14 + [8200, 17] + [9100] * 16, [1] * 31 + [0])):
        x = Weighed(H, Hkv, hd, kind, ctx, ks, 6)
        assert x.weigh() == 0
        x.check_weights()


@pytest.mark.parametrize("H,Hkv,hd,kind", [(8, 2, 128, "f16"), (4, 4, 64, "f16"), (4, 2, 64, "f32")])
@pytest.mark.parametrize("ctx,ks", [([300, 40], [3, 0]), ([0], [400])], ids=str)
@pytest.mark.parametrize("far", [False, True])
def test_large_references(H, Hkv, hd, kind, ctx, ks, far):
    """Scores so far apart that a row's weight is all on the keys that attain its largest, in equal shares; the statistics are the attention's own."""
    x = Weighed(H, Hkv, hd, kind, ctx, ks, 9)
    g = np.random.default_rng(9)
    for b in range(len(ks)):
        n = x.tot[b]
        k = torch.tensor(g.integers(1, 9, (n, Hkv)) * (4096.0 if far else 1.0), device="cuda")[:, :, None].expand(n, Hkv, hd)
        p = torch.arange(n, device="cuda")
        blk = torch.from_numpy(x.full[b].astype(np.int64)).cuda()[p // 16]
        x.kp[blk, :, :, p % 16] = k.reshape(n, Hkv, hd // 8, 8).to(x.kp.dtype)
    x.q.fill_(64.0 if not far else 65504.0 if kind == "f16" else 2.0 ** 40)
    _, status = x.run(stats=x.stats)
    assert status == 0 and (x.stats[:, :, 0].abs() >= (2.0 ** 24 if far else 500)).all()
    assert x.weigh() == 0
    for b in range(len(ks)):
        k, _ = x.dense(b)
        seen = x.visible(b)
        for h in range(Hkv):
            s = k[:, h, 0].double().expand(len(seen), -1).masked_fill(~seen, -math.inf)
            p = (s == s.amax(dim=1, keepdim=True)).double()
            want = (p / p.sum(dim=1, keepdim=True)).sum(dim=0) * (H // Hkv)
            want[:x.ctx[b]] += x.mass0[0, b, h, :x.ctx[b]].double()
            # Ties are equal whatever the roundings: what is left are the sums and the quotients.  Below 2^24 the fp16 attention takes c s - m in one
            # rounding, which of the largest score is the rounding of m = c s and not 0: at most 2^-24 of m < 2^15, so that its probability is within
            # 2^-9 of 1, and is off by half a step, 2^-11, as the sum l has it (fp16) and as it is here (not rounded).
            tol = (len(seen) * (H // Hkv) + x.tot[b] + 64) * 2.0 ** -23 + (2.0 ** -11 if kind == "f16" and not far else 0)
            assert ((x.ledger.mass[0, b, h, :x.tot[b]].double() - want).abs() <= want * tol).all()


def test_rows_without_statistics_give_nothing():
    x = Weighed(8, 2, 128, "f16", [100, 20], [3, 2], 7)
    x.weigh()
    whole = x.ledger.mass.clone()
    for bad in ((0.0, 0.0), (float("nan"), 1.0), (0.0, float("nan")), (float("inf"), 1.0), (float("-inf"), 0.0), (0.0, float("inf"))):
        keep = x.stats.clone()
        x.stats[1, :, 0], x.stats[1, :, 1] = bad
        assert x.weigh() == 0
        assert torch.isfinite(x.ledger.mass).all()
        assert (x.ledger.mass[0, 0, :, :102] <= whole[0, 0, :, :102]).all() and torch.equal(x.ledger.mass[0, 1], whole[0, 1])
        x.stats.copy_(keep)
    # a key that is not a number: its own weight, where somebody's statistics hide it, and no other's
    x.kp[int(x.full[0, 2]), 1, 3, 4, 5] = float("nan")
    assert x.weigh() == 0
    odd = torch.isnan(x.ledger.mass)
    assert odd.sum() <= 1 and torch.equal(x.ledger.mass[~odd & (torch.arange(x.width, device="cuda") != 36)], whole[~odd & (torch.arange(x.width, device="cuda") != 36)])


@pytest.mark.parametrize("H,Hkv,hd,kind,ctx,ks", [
    (64, 8, 128, "f16", [300, 40, 5], [0, 1, 2]), (40, 40, 128, "f16", [100, 33], [0, 15]), (12, 12, 64, "f16", [70, 64], [0, 4]), (6, 2, 64, "f16", [50, 9], [3, 19]),
    (16, 2, 128, "f16", [9000], [8]), (8, 2, 128, "f16", [60, 5], [100, 15]), (12, 12, 64, "f16", [20, 100], [79, 128]), (40, 40, 128, "f16", [700] * 8, [200] * 8),
    (64, 8, 64, "f16", [900, 9] * 20, [150, 11] * 20), (4, 2, 64, "f32", [40, 7], [2, 9]), (8, 2, 128, "f32", [100], [50]), (8, 8, 8, "f32", [33, 4], [0, 90]),
    (8, 2, 256, "f16", [50, 60], [0, 30]), (8, 8, 32, "f16", [64], [3])], ids=str)
def test_infinite_keys_that_no_row_looks_at_weigh_nothing(H, Hkv, hd, kind, ctx, ks):
    """An infinity in a key whose every score is minus infinity is a key with a score of -10^4: no weight, and the others as they were, whatever the number
    of rows (multiples of 16 and others, of a KV head, in every kernel)."""
    x = Weighed(H, Hkv, hd, kind, ctx, ks, 12)
    low, high = 3, hd - 2                                           # elements that all queries have below -1, above 1
    x.q[:, :, low], x.q[:, :, high] = -1 - x.q[:, :, low].abs(), 1 + x.q[:, :, high].abs()

    def plant(value):
        for b, c in enumerate(ctx):
            for slot, e, v in ((1, low, value), (c, high, -value), (x.tot[b] - 1, low, value)):   # behind all rows, the first row's, the last row's
                x.kp[int(x.full[b, slot // 16]), :, e // 8, slot % 16, e % 8] = v
    plant(60000.0)
    _, status = x.run(stats=x.stats)
    assert status == 0 and x.weigh() == 0
    mass, born, stats = x.ledger.mass.clone(), x.ledger.born.clone(), x.stats.clone()
    plant(math.inf)
    _, status = x.run(stats=x.stats)
    assert status == 0 and torch.equal(x.stats, stats)
    assert x.weigh() == 0
    assert torch.isfinite(x.ledger.mass).all() and torch.equal(x.ledger.mass, mass) and torch.equal(x.ledger.born, born)
    for b, c in enumerate(ctx):
        assert torch.equal(x.ledger.mass[0, b, :, 1], x.mass0[0, b, :, 1]) and (x.ledger.mass[0, b, :, [c, x.tot[b] - 1]] == 0).all()


def test_damage_is_left_out_of_the_weights():
    from paper_2402_15678_amd import binding, harness
    x = Weighed(8, 2, 128, "f16", [100, 20, 40], [3, 2, 0], 8)
    good = x.table.copy()
    x.table[0, 3] = 1 << 30
    assert x.weigh() == binding.MN_DEV_BLOCK_TABLE
    x.table = good
    x.check_weights(lost=[(0, slice(48, 64))])
    for ctx, n, flag in (([100, -1, 40], None, binding.MN_DEV_CTX), ([100, x.max_ctx, 40], None, binding.MN_DEV_CTX), ([104, 2, 41], [4, 3, 1], binding.MN_DEV_CTX),
                         ([104, 24, 41], [4, 4, 1], binding.MN_DEV_SPEC_LEN)):
        kv = harness.DeviceKV(x.d, x.bs, x.kp.shape[0], x.table, ctx, [x.kp], [x.vp])
        assert x.weigh(kv=kv, n_out=n) == flag
        x.check_weights(seqs=[0, 2])
    for spec in ([3, 2, 1], [4, 1, -1], [4, 2, 0]):
        assert x.weigh(spec=spec) == binding.MN_DEV_SPEC_LEN
        assert torch.equal(x.ledger.mass, x.mass0) and torch.equal(x.ledger.born, x.born0)


# --------------------------------------------------------------------------------------------------------------
# eviction
# --------------------------------------------------------------------------------------------------------------

class Cache:
    """Slots with n[s] tokens each in `layers` layers; every token's rows are random; blocks scattered."""

    def __init__(self, Hkv, hd, kind, layers, n, seed, bs=16, width=None, spare=3, H=None):
        from paper_2402_15678_amd import harness
        self.n, self.bs, self.layers, self.Hkv = list(n), bs, layers, Hkv
        r = np.random.default_rng(seed)
        need = [-(-x // bs) for x in n]
        nb = sum(need) + spare
        ids = r.permutation(nb).astype(np.int32)
        self.table = np.full((len(n), max(max(need), 1) + 1), -1, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = ids[at:at + m]
            at += m
        self.d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if kind == "f16" else synth.DT_F32, layers, 128, H or Hkv, Hkv, hd, 128, 8, 1 << 20)
        if (self.d.n_heads * hd) % 128:
            self.d = synth.ModelDesc(synth.ARCH_LLAMA, self.d.dtype, layers, 128, Hkv * 16, Hkv, hd, 128, 8, 1 << 20)
        self.model = harness.DeviceModel.random_on_device(self.d, 1)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.k = torch.randn((layers, nb, Hkv, hd // 8, bs, 8), generator=g, device="cuda").to(DT[kind])
        self.v = torch.randn((layers, nb, Hkv, hd, bs), generator=g, device="cuda").to(DT[kind])
        self.kv = harness.DeviceKV(self.d, bs, nb, self.table, n, list(self.k), list(self.v))
        self.pool = harness.KVPool.from_tables(self.model, self.kv)
        self.width = width or max(n) + 5
        shape = (layers, len(n), Hkv, self.width)
        self.mass = torch.exp(torch.randn(shape, generator=g, device="cuda") * 2)
        self.born = torch.arange(self.width, dtype=torch.int32, device="cuda").expand(shape).contiguous()
        self.ledger = harness.KVLedger(self.model, self.kv, self.mass, self.born)

    def snapshot(self):
        return dict(k=self.k.clone(), v=self.v.clone(), mass=self.mass.cpu().numpy().copy(), born=self.born.cpu().numpy().copy(),
                    table=self.kv.block_tables.cpu().numpy().copy(), refs=self.pool.block_refs.cpu().numpy().copy(),
                    held=self.pool.seq_blocks.cpu().numpy().copy(), ctx=self.kv.ctx_lens.cpu().numpy().copy())

    def evict(self, keep, sinks, recent):
        self.pool.dev_status.zero_()
        self.pool.evict(torch.tensor(keep, dtype=torch.int32, device="cuda"), sinks, recent, self.ledger)
        torch.cuda.synchronize()
        return self.pool.dev_status.item()

    def want(self, s, keep, sinks, recent, skip=()):
        """The snapshot s after the eviction, by lists."""
        for b, kp in enumerate(keep):
            n = int(s["ctx"][b])
            if kp < 0 or kp >= n or b in skip:
                continue
            for layer in range(self.layers):
                for h in range(self.Hkv):
                    m, o = s["mass"][layer, b, h], s["born"][layer, b, h]
                    last = int(o[:n].max())
                    order = sorted(range(n), key=lambda i: (0 if i < sinks or o[i] > last - recent else 1 if m[i] == m[i] else 2, 0.0 if m[i] != m[i] or
                                                            i < sinks or o[i] > last - recent else -float(m[i]), i))
                    stay = set(order[:kp])
                    holes, movers = [i for i in range(kp) if i not in stay], [i for i in range(kp, n) if i in stay]
                    assert len(holes) == len(movers)
                    if not holes:
                        continue
                    at = lambda ii: (torch.tensor([int(s["table"][b, i // self.bs]) for i in ii]).cuda(), torch.tensor([i % self.bs for i in ii]).cuda())  # noqa: E731
                    (tb, to), (fb, fo) = at(holes), at(movers)
                    s["k"][layer][tb, h, :, to] = s["k"][layer][fb, h, :, fo]
                    s["v"][layer][tb, h, :, to] = s["v"][layer][fb, h, :, fo]
                    m[holes], o[holes] = m[movers], o[movers]
            now = -(-kp // self.bs)
            for i in range(now, int(s["held"][b])):
                s["refs"][s["table"][b, i]] -= 1
                s["table"][b, i] = -1
            s["held"][b], s["ctx"][b] = now, kp
        return s

    def check(self, s):
        assert torch.equal(self.k, s["k"]) and torch.equal(self.v, s["v"])
        for key, t in (("mass", self.mass), ("born", self.born), ("table", self.kv.block_tables), ("refs", self.pool.block_refs),
                       ("held", self.pool.seq_blocks), ("ctx", self.kv.ctx_lens)):
            assert np.array_equal(t.cpu().numpy(), s[key], equal_nan=key == "mass"), key


@pytest.mark.parametrize("Hkv,hd,kind,layers,bs", [(8, 128, "f16", 3, 16), (12, 64, "f16", 2, 16), (4, 64, "f32", 2, 16), (2, 256, "f32", 1, 16), (8, 8, "f32", 2, 16),
                                                   (2, 128, "f16", 2, 5), (2, 32, "f32", 2, 48), (1, 16, "f32", 1, 1)])
@pytest.mark.parametrize("n,keep,sinks,recent", [([100, 64, 1, 0, 65], [64, 64, 64, 64, 64], 4, 16), ([300, 17, 40], [16, 1, 39], 0, 0), ([300, 300, 300], [-1, 0, 299], 3, 1),
                                                 ([700, 129], [513, 128], 20, 100), ([50, 60], [7, 12], 9, 30)], ids=str)
def test_eviction_matches_the_lists(Hkv, hd, kind, layers, bs, n, keep, sinks, recent):
    x = Cache(Hkv, hd, kind, layers, n, Hkv + hd, bs=bs)
    s = x.snapshot()
    assert x.evict(keep, sinks, recent) == 0
    x.check(x.want(s, keep, sinks, recent))


@pytest.mark.parametrize("Hkv,hd,kind", [(2, 128, "f32"), (2, 256, "f16"), (3, 32, "f16"), (1, 8, "f16")])
@pytest.mark.parametrize("n,keep,sinks,recent", [([100, 64, 1, 65], [64, 63, 64, 64], 4, 16), ([300, 17], [16, 1], 0, 0), ([700, 129], [513, 128], 20, 100)], ids=str)
def test_pages_of_every_size_are_evicted(Hkv, hd, kind, n, keep, sinks, recent):
    """Pages of 256 bytes, 1 KB and 8 KB: what a wave takes in part of one turn, in one, and in two."""
    x = Cache(Hkv, hd, kind, 2, n, Hkv + hd)
    s = x.snapshot()
    assert x.evict(keep, sinks, recent) == 0
    x.check(x.want(s, keep, sinks, recent))


@pytest.mark.parametrize("n", [1000, 4096, 5000, 9000, 20000])
def test_long_contexts_are_evicted_again_and_again(n):
    """By half, by one, by a few, and to the last protected one."""
    x = Cache(2, 64, "f16", 1, [n, n // 3], 1)
    for keep in ([n // 2, -1], [n // 2 - 1, n // 3 - 1], [n // 2 - 9, n // 4], [40, 40], [12, 3]):
        s = x.snapshot()
        assert x.evict(keep, 4, 32) == 0
        x.check(x.want(s, keep, 4, 32))
        x.mass.copy_(torch.rand_like(x.mass))


def test_equal_weights_infinities_zeros_and_no_numbers():
    x = Cache(4, 64, "f16", 2, [200, 333, 90], 2)
    x.mass[0] = 1.0
    x.mass[1, 0, :, ::3] = float("inf")
    x.mass[1, 0, 1] = float("nan")
    x.mass[1, 1] = torch.where(torch.rand_like(x.mass[1, 1]) < 0.5, 0.0, -0.0)
    x.mass[1, 2, :, 10:] = -torch.arange(x.width - 10, device="cuda", dtype=torch.float32)
    x.mass[1, 2, :, 50] = float("-inf")
    for keep in ([150, 111, 80], [20, 64, 41], [5, 5, 5]):
        s = x.snapshot()
        assert x.evict(keep, 2, 7) == 0
        x.check(x.want(s, keep, 2, 7))


def test_sharers_and_damage_are_left_alone():
    from paper_2402_15678_amd import binding
    x = Cache(2, 64, "f16", 2, [200, 150, 60, 0, 90], 3)
    x.pool.fork(torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"))
    x.mass[:, 3], x.born[:, 3] = x.mass[:, 0], x.born[:, 0]
    s = x.snapshot()
    assert x.evict([100, 100, -1, 100, 80], 4, 16) == binding.MN_DEV_SHARED
    x.check(x.want(s, [100, 100, -1, 100, 80], 4, 16, skip=(0, 3)))
    # what they share lies within the first tokens, or behind the new end
    s = x.snapshot()
    assert x.evict([100, -1, -1, -1, -1], 96, 3) == binding.MN_DEV_SHARED
    x.check(s)
    s = x.snapshot()
    assert x.evict([112, -1, -1, -1, -1], 112, 16) == 0
    x.check(x.want(s, [112, -1, -1, -1, -1], 112, 16))
    good, held, ctx = x.kv.block_tables.clone(), x.pool.seq_blocks.clone(), x.kv.ctx_lens.clone()
    for damage, flag in ((lambda: x.kv.block_tables.__setitem__((2, 1), 1 << 30), binding.MN_DEV_BLOCK_TABLE), (lambda: x.kv.block_tables.__setitem__((2, 3), -1), binding.MN_DEV_BLOCK_TABLE),
                         (lambda: x.pool.seq_blocks.__setitem__(2, 3), binding.MN_DEV_BLOCK_TABLE), (lambda: x.pool.seq_blocks.__setitem__(2, 1000), binding.MN_DEV_BLOCK_TABLE),
                         (lambda: x.kv.ctx_lens.__setitem__(2, x.width + 1), binding.MN_DEV_CTX)):
        damage()
        s = x.snapshot()
        assert x.evict([-1, 70, 40, -1, 60], 4, 16) == flag
        x.check(x.want(s, [-1, 70, 40, -1, 60], 4, 16, skip=(2,)))
        x.kv.block_tables[2], x.pool.seq_blocks[2], x.kv.ctx_lens[2] = good[2], held[2], ctx[2]


def test_a_shared_block_among_the_first_tokens_is_no_hindrance():
    """All that stays are first tokens: nothing moves, and who shares their blocks goes on reading them; the next token gets a block of its own."""
    x = Cache(2, 64, "f16", 2, [200, 0], 13)
    x.pool.fork(torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"))
    x.mass[:, 1], x.born[:, 1] = x.mass[:, 0], x.born[:, 0]
    s = x.snapshot()
    assert x.evict([90, -1], 100, 3) == 0                           # blocks 0 .. 5 stay, the last with 10 tokens; the first 100 tokens are in blocks 0 .. 6
    x.check(x.want(s, [90, -1], 100, 3))
    x.pool.reserve(torch.tensor([91, 0], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    table = x.kv.block_tables.tolist()
    assert x.pool.dev_status.item() == 0 and table[0][:5] == table[1][:5] and table[0][5] != table[1][5] and x.pool.block_refs[table[0][5]].item() == 1
    assert torch.equal(x.k[:, table[0][5]], x.k[:, table[1][5]]) and torch.equal(x.v[:, table[0][5]], x.v[:, table[1][5]])


def test_more_layers_than_a_launch_holds():
    x = Cache(1, 16, "f32", 100, [60, 33], 4)
    s = x.snapshot()
    assert x.evict([31, 20], 2, 5) == 0
    x.check(x.want(s, [31, 20], 2, 5))


def test_evictions_are_captured_and_replayed():
    x = Cache(4, 64, "f16", 2, [300, 120], 5)
    start = x.snapshot()
    state, mass, born, k, v = x.pool.state.clone(), x.mass.clone(), x.born.clone(), x.k.clone(), x.v.clone()
    keep = torch.tensor([100, 100], dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        x.pool.evict(keep, 4, 8, x.ledger)                          # (its workspace)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            x.pool.evict(keep, 4, 8, x.ledger)
        for budget in ([100, 100], [64, 120], [7, 3]):
            for t, old in ((x.pool.state, state), (x.mass, mass), (x.born, born), (x.k, k), (x.v, v)):
                t.copy_(old)
            keep.copy_(torch.tensor(budget, dtype=torch.int32))
            g.replay()
            stream.synchronize()
            s = {key: (t.clone() if torch.is_tensor(t) else t.copy()) for key, t in start.items()}
            x.check(x.want(s, budget, 4, 8))
    torch.cuda.current_stream().wait_stream(stream)


# --------------------------------------------------------------------------------------------------------------
# all of it together
# --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("H,Hkv,hd,kind", [(8, 2, 128, "f16"), (12, 12, 64, "f16"), (4, 2, 64, "f32")])
def test_a_life_in_a_bounded_cache(H, Hkv, hd, kind):
    """Prompts enter, steps of several tokens follow of which some are accepted, and whenever a request holds more than its budget it is cut
    back.  Every step's attention is checked against the definition on the tokens that each head should still hold, which a plain model keeps as
    dense rows, and the ledger against that model."""
    from paper_2402_15678_amd import harness
    torch.manual_seed(1)
    B, budget, sinks, recent, bs, steps = 3, 60, 3, 20, 16, 6
    r = np.random.default_rng(7)
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if kind == "f16" else synth.DT_F32, 1, 128, H, Hkv, hd, 128, 8, 1 << 16)
    model = harness.DeviceModel.random_on_device(d, 1)
    width, nb = 10, 30
    kv = harness.DeviceKV(d, bs, nb, np.full((B, width), -1, np.int32), [0] * B,
                          [torch.zeros((nb, Hkv, hd // 8, bs, 8), dtype=DT[kind], device="cuda")], [torch.zeros((nb, Hkv, hd, bs), dtype=DT[kind], device="cuda")])
    pool = harness.KVPool.from_tables(model, kv)
    ledger = harness.KVLedger.empty(model, kv, B, width * bs)
    rule = harness.RowRule(hd, [hd // 2], 10000.0, 1 + 0.1 * torch.randn(hd, device="cuda"), 1 + 0.1 * torch.randn(hd, device="cuda"))
    rows_of = harness.WindowSession(model, kv, B, 400, 140, width * bs, width * bs, 0)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    # the plain model: per sequence and KV head the rows (k, v, mass, born) of the tokens held
    held = [[[] for _ in range(Hkv)] for _ in range(B)]
    seen = [0] * B
    for step in range(steps):
        ks = [int(r.integers(70, 130)) for _ in range(B)] if step == 0 else [int(r.integers(0, 9)) for _ in range(B)]
        ctx = kv.ctx_lens.tolist()
        pool.reserve(i32([c + k + 1 for c, k in zip(ctx, ks)]))
        M, spec = sum(ks) + B, i32(ks)
        qkv = torch.randn((M, (H + 2 * Hkv) * hd), device="cuda")
        q, k, v = qkv[:, :H * hd].view(M, H, hd), qkv[:, H * hd:(H + Hkv) * hd].view(M, Hkv, hd), qkv[:, (H + Hkv) * hd:].view(M, Hkv, hd)
        place = i32(np.concatenate([np.arange(s, s + k_ + 1) for s, k_ in zip(seen, ks)]).tolist()).view(1, M)
        q_out, k_out, v_out = (torch.zeros((M, h * hd), dtype=DT[kind], device="cuda") for h in (H, Hkv, Hkv))
        harness.qk_norm_rope(model, q, k, v, rule, place, spec, ks, q_out, kv=kv, k_out=k_out, v_out=v_out, dev_status=pool.dev_status)
        out, stats = torch.zeros((M, H * hd), dtype=DT[kind], device="cuda"), torch.zeros((M, H, 2), device="cuda")
        qd = q_out.view(M, H, hd)
        rows_of.attention(qd, spec, ks, out, stats=stats)
        took = [k_ + 1 if step == 0 else int(r.integers(1, k_ + 2)) for k_ in ks]
        kv.ctx_lens.add_(i32(took))                                 # (what mn_accept_and_commit does)
        ledger.weigh(qd, stats, spec, ks, 0, width * bs, i32(took), i32(seen))
        torch.cuda.synchronize()
        assert pool.dev_status.item() == 0 and rows_of.dev_status.item() == 0 and ledger.dev_status.item() == 0
        mass, born = ledger.mass.cpu(), ledger.born.cpu()
        a = 0
        for b in range(B):
            n, G = ks[b] + 1, H // Hkv
            for h in range(Hkv):
                own = [(k_out[a + j].view(Hkv, hd)[h], v_out[a + j].view(Hkv, hd)[h]) for j in range(n)]
                kk = torch.stack([t[0] for t in held[b][h]] + [t[0] for t in own])[:, None]
                vv = torch.stack([t[1] for t in held[b][h]] + [t[1] for t in own])[:, None]
                want, bound = attend(qd[a:a + n, h * G:(h + 1) * G], kk, vv, torch.arange(ctx[b], ctx[b] + n, device="cuda"), kind == "f16")
                check(out[a:a + n].view(n, H, hd)[:, h * G:(h + 1) * G].reshape(n, -1), want, bound)
                # (the library's weights are within their own tests' bounds; here: which token has them)
                for i, t in enumerate(held[b][h]):
                    t[2] = float(mass[0, b, h, i])
                    assert int(born[0, b, h, i]) == t[3]
                for j in range(took[b]):
                    assert int(born[0, b, h, ctx[b] + j]) == seen[b] + j
                    held[b][h].append([own[j][0], own[j][1], float(mass[0, b, h, ctx[b] + j]), seen[b] + j])
            seen[b] += took[b]
            a += n
        if step == 0:
            for b in range(B):                                      # of a prompt the weights of all rows add up to their number
                total = ledger.mass[0, b, :, :took[b]].double().sum(dim=1)
                assert ((total - took[b] * (H // Hkv)).abs() <= took[b] * (H // Hkv) * 2.0 ** -9).all()
        pool.evict(i32([budget] * B), sinks, recent, ledger)
        torch.cuda.synchronize()
        assert pool.dev_status.item() == 0
        for b in range(B):
            for h in range(Hkv):
                t = held[b][h]
                if len(t) <= budget:
                    continue
                last = max(x[3] for x in t)
                order = sorted(range(len(t)), key=lambda i: (0 if i < sinks or t[i][3] > last - recent else 1, 0 if i < sinks or t[i][3] > last - recent else -t[i][2], i))
                stay = set(order[:budget])
                holes, movers = [i for i in range(budget) if i not in stay], [i for i in range(budget, len(t)) if i in stay]
                for i, j in zip(holes, movers):
                    t[i] = t[j]
                held[b][h] = t[:budget]
        assert kv.ctx_lens.tolist() == [len(held[b][0]) for b in range(B)]
        assert pool.seq_blocks.tolist() == [max(-(-len(held[b][0]) // bs), 0) if len(held[b][0]) == budget else pool.seq_blocks[b].item() for b in range(B)]


@pytest.mark.parametrize("H,Hkv,hd,kind,lens", [(8, 2, 128, "f16", (3, 0, 8)), (12, 12, 64, "f16", (20, 1, 70)), (4, 2, 64, "f32", (4, 2, 0)), (8, 2, 256, "f16", (9, 0, 1))], ids=str)
def test_steps_are_captured_and_replayed(H, Hkv, hd, kind, lens):
    """Room, rows, attention, commit, weights and eviction of a step in one graph: replayed over changing contexts it leaves, bit for bit, what the calls leave
    that are made one by one."""
    from paper_2402_15678_amd import harness
    B, budget, bs, nb, width, steps = len(lens), 90, 16, 40, 12, 5
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if kind == "f16" else synth.DT_F32, 1, 128, H, Hkv, hd, 128, 8, 1 << 16)
    model, M = harness.DeviceModel.random_on_device(d, 1), sum(lens) + B
    ctx0 = [70, 0, 88]
    table = np.full((B, width), -1, np.int32)
    for b, c in enumerate(ctx0):
        table[b, :-(-c // bs)] = np.arange(-(-c // bs)) + 6 * b
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    k0, v0 = draw(nb, Hkv, hd // 8, bs, 8).to(DT[kind]), draw(nb, Hkv, hd, bs).to(DT[kind])
    kv = harness.DeviceKV(d, bs, nb, table, ctx0, [k0.clone()], [v0.clone()])
    pool = harness.KVPool.from_tables(model, kv)
    ledger = harness.KVLedger.empty(model, kv, B, width * bs)
    ledger.mass.copy_(torch.rand(ledger.mass.shape, generator=g, device="cuda"))
    ledger.born.copy_(torch.arange(width * bs, dtype=torch.int32, device="cuda").expand(ledger.born.shape))
    rule = harness.RowRule(hd, [hd // 2], 10000.0, 1 + 0.1 * draw(hd), 1 + 0.1 * draw(hd))
    ses = harness.WindowSession(model, kv, B, M, max(lens) + 1, width * bs, width * bs, 0)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    qkv, place, took, seen, spec, keep = draw(M, H + 2 * Hkv, hd), i32([[0] * M]), i32([0] * B), i32(ctx0), i32(lens), i32([budget] * B)
    room = i32([0] * B)
    q, out, stats = (torch.zeros(s, dtype=t, device="cuda") for s, t in (((M, H, hd), DT[kind]), ((M, H * hd), DT[kind]), ((M, H, 2), torch.float32)))

    def step():
        torch.add(kv.ctx_lens, spec, out=room)
        room.add_(1)
        pool.reserve(room)
        harness.qk_norm_rope(model, qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], rule, place, spec, lens, q, kv=kv, dev_status=pool.dev_status)
        ses.attention(q, spec, lens, out, stats=stats)
        kv.ctx_lens.add_(took)
        ledger.weigh(q, stats, spec, lens, 0, width * bs, took, seen)
        seen.add_(took)
        pool.evict(keep, 3, 20, ledger)
    state = (kv.k_pages[0], kv.v_pages[0], ledger.mass, ledger.born, pool.state, seen, q, out, stats)
    start = [t.clone() for t in state]
    r = np.random.default_rng(4)
    inputs = [(draw(M, H + 2 * Hkv, hd), [int(r.integers(0, 5000)) for _ in range(M)], [int(r.integers(1, k + 2)) for k in lens]) for _ in range(steps)]

    def run(go):
        for t, old in zip(state, start):
            t.copy_(old)
        left, ctx = [], list(ctx0)
        for rows, at, n in inputs:
            qkv.copy_(rows)
            place.copy_(i32([at]))
            took.copy_(i32(n))
            go()
            torch.cuda.synchronize()
            assert pool.dev_status.item() == 0 and ses.dev_status.item() == 0 and ledger.dev_status.item() == 0
            held = [-(-(c + k + 1) // bs) for c, k in zip(ctx, lens)]  # (a slot keeps the room of rows that were not accepted)
            held = [max(h, o) for h, o in zip(held, left[-1][1])] if left else held
            ctx = [c + m for c, m in zip(ctx, n)]
            held = [-(-budget // bs) if c > budget else h for c, h in zip(ctx, held)]
            ctx = [min(c, budget) for c in ctx]
            assert kv.ctx_lens.tolist() == ctx and pool.seq_blocks.tolist() == held
            left.append(([t.clone() for t in state], held))
        return left
    want = run(step)
    assert max(want[-1][0][5].tolist()) > budget                    # (somebody was cut back)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for a, b in zip(run(graph.replay), want):
        for x, y in zip(a[0], b[0]):
            assert torch.equal(x, y)
