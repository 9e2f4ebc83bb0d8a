"""What the operators of a bounded paged cache cost: the rows of a projection made ready for it, attention that looks back a
window and at a few first tokens, the weight that attention has given to every cached token, and the eviction that goes by it.

A serving program meets them in this order: a step's or a prompt's projected rows are normed per head, turned to their positions
and put into the cache (``rows``); its queries attend to the last tokens and the first few (``window``), prompts and chunks of
them as well as single tokens; or they see everything and the weights that they gave are added up per cached token (``weigh``),
until the cache is cut back to the tokens that matter (``evict``).

``own`` false: plain torch, 32 bits (64 for angles).  ``own`` true: the library's entry points.  Head geometries are those of the
repository's model descriptions (64/8 x 128, 40 x 128, 12 x 64 in 16 bits, 4 x 64 in 32) and a few generic ones; cached rows
are N(0, 1), pages are scattered at random over the pool.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

BLOCK = 16
LOG2E = 1.4426950408889634
H70B, H13B, HSSM, HTINY = (64, 8, 128, "f16"), (40, 40, 128, "f16"), (12, 12, 64, "f16"), (4, 4, 64, "f32")
GEOMETRIES = (H70B, H70B, H13B, H13B, HSSM, HTINY, (32, 4, 128, "f16"), (16, 2, 64, "f16"), (8, 8, 32, "f16"),
              (8, 2, 256, "f16"), (8, 2, 128, "f32"))


# --------------------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------------------

def _case(op, g, batch, lo, hi, k_lo, k_hi, shape_seed, **more):
    """`lo` .. `hi`: cached tokens of a sequence; `k_lo` .. `k_hi`: rows of a sequence behind its first one.  A prompt has
    `lo` = `hi` = 0 and all its tokens as rows."""
    return dict(heads=g[0], kv_heads=g[1], head_dim=g[2], dtype=g[3], op=op, batch=batch, lo=lo, hi=hi, k_lo=k_lo, k_hi=k_hi,
                shape_seed=shape_seed, **more)


def _rows(g, batch, lo, hi, k_lo, k_hi, seed, wide, norm, rot, axes):
    """`wide`: rows of 32 bits, as the projection leaves them; else of the cache's type.  `rot`: turned elements of a head."""
    return _case("rows", g, batch, lo, hi, k_lo, k_hi, seed, wide=wide, norm=norm, rot=rot, axes=axes)


def _window(g, batch, lo, hi, k_lo, k_hi, seed, window, sinks):
    return _case("window", g, batch, lo, hi, k_lo, k_hi, seed, window=window, sinks=sinks)


def _weigh(g, batch, lo, hi, k_lo, k_hi, seed, committed):
    """`committed`: a random number of each sequence's rows has been accepted and counts; else all do."""
    return _case("weigh", g, batch, lo, hi, k_lo, k_hi, seed, committed=committed)


def _evict(g, layers, batch, lo, hi, seed, keep, sinks, recent, again):
    """`keep`: tokens that stay; `again`: an earlier eviction has left the tokens out of order."""
    return _case("evict", g, batch, lo, hi, 0, 0, seed, layers=layers, keep=keep, sinks=sinks, recent=recent, again=again)


def listed():
    named = lambda name, c: dict(c, name=name)  # noqa: E731
    return [
        # one token each on a drafting model: launch and latency count
        named("rows-ssm-b4-decode", _rows(HSSM, 4, 50, 900, 0, 0, 1, False, True, 64, 1)),
        # a full server's verification step, straight behind the projection
        named("rows-70b-b64-k8", _rows(H70B, 64, 200, 2000, 8, 8, 2, True, True, 128, 1)),
        # prompts with positions in time, height and width
        named("rows-70b-b4-prompts-3-axes", _rows(H70B, 4, 0, 0, 500, 3000, 3, False, True, 128, 3)),
        # the smallest windowed step: three short requests of a small fp32 model
        named("window-tiny-fp32-b3-k4", _window(HTINY, 3, 20, 120, 4, 4, 4, 48, 4)),
        # streaming: one token each for 24 long conversations
        named("window-70b-b24-decode", _window(H70B, 24, 500, 30000, 0, 0, 5, 4096, 4)),
        # ragged prompts, most keys out of sight
        named("window-13b-b4-prompts", _window(H13B, 4, 0, 0, 1500, 6000, 6, 1024, 16)),
        # long inputs fed in pieces: a piece of each behind what is cached
        named("window-70b-b2-chunk", _window(H70B, 2, 6000, 20000, 1500, 2500, 7, 8192, 64)),
        # a drafting model's step
        named("weigh-ssm-b2-decode", _weigh(HSSM, 2, 100, 400, 0, 0, 8, False)),
        # a verification step after its acceptance
        named("weigh-70b-b32-k8", _weigh(H70B, 32, 1000, 8000, 8, 8, 9, True)),
        # prompts: every token's weight in the eyes of those behind it
        named("weigh-13b-b2-prompts", _weigh(H13B, 2, 0, 0, 1000, 3000, 10, False)),
        # one short request cut back: bookkeeping and latency
        named("evict-tiny-b1", _evict(HTINY, 2, 1, 100, 100, 11, 64, 4, 16, False)),
        # a server cut back to a budget, not for the first time
        named("evict-70b-b16", _evict(H70B, 8, 16, 1000, 4000, 12, 1024, 4, 256, True)),
    ]


def _log_int(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    g = rng.choice(GEOMETRIES)
    h, hk, hd, dtype = g
    seed = rng.randrange(1 << 20)
    span = lambda lo, hi: sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))  # noqa: E731
    slow = 4 if dtype == "f32" or hd not in (64, 128) else 1
    pick = rng.randrange(4)
    if pick == 3:
        layers, batch = rng.randint(1, 8), _log_int(rng, 1, 16)
        lo, hi = span(16, 4000 * H70B[1] * 128 // max(hk * hd, H70B[1] * 128))
        case = _evict(g, layers, batch, lo, hi, seed, 0, rng.randint(0, 8), 0, rng.random() < 0.5)
        longest = max(_shape(case)[0])
        # the longest one down to half of it, or by a token or a few
        case["keep"] = max(1, rng.randint(longest // 2, longest - 1) if rng.random() < 0.5 else longest - rng.randint(1, 9))
        case["recent"] = rng.randint(1, max(1, case["keep"] // 4))
        return case
    batch = _log_int(rng, 1, 32)
    prompts = rng.random() < 0.4
    if pick == 0:
        rot = hd if rng.random() < 0.7 else hd // 2
        axes = rng.choice((1, 1, 2, 3))
        if prompts:
            lo, hi, k_lo, k_hi = 0, 0, *span(1, max(2, min(3000, 5000 * 80 * 128 // (batch * (h + 2 * hk) * hd))))
        else:
            (lo, hi), (k_lo, k_hi) = span(1, 2000), sorted((rng.randint(0, 12), rng.randint(0, 12)))
        return _rows(g, batch, lo, hi, k_lo, k_hi, seed, rng.random() < 0.5, rng.random() < 0.7, rot, axes)
    # pairs of a row and a key, and cached elements, at most those of the operator's largest listed case
    pairs, cached = ((1 << 25, 1 << 28) if pick == 1 else (1 << 22, 1 << 27))
    pairs = pairs * 40 * 128 // (h * hd) // slow
    if prompts:
        batch = min(batch, 8)
        lo, hi, k_lo, k_hi = 0, 0, *span(1, max(2, min(6000, int(math.sqrt(pairs / batch)))))
    else:
        k_lo, k_hi = sorted((rng.randint(0, 12), rng.choice((0, 12, 200))))
        lo, hi = span(1, max(2, min(20000, pairs // (batch * (k_hi + 1)), cached // (batch * hk * hd))))
    if pick == 1:
        return _window(g, batch, lo, hi, k_lo, k_hi, seed, _log_int(rng, 1, 8192), rng.choice((0, rng.randint(1, 80))))
    return _weigh(g, batch, lo, hi, k_lo, k_hi, seed, rng.random() < 0.5)


def _shape(case):
    """Cached tokens and rows behind the first one, per sequence, from the case alone."""
    r = random.Random(case["shape_seed"])
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    return n, [r.randint(case["k_lo"], case["k_hi"]) for _ in range(case["batch"])]


def _committed(case):
    """Accepted rows per sequence, or all."""
    _, ks = _shape(case)
    r = random.Random(case["shape_seed"] + 1)
    return [r.randint(1, k + 1) if case["committed"] else k + 1 for k in ks]


def _axis_pairs(case):
    pairs, n = case["rot"] // 2, case["axes"]
    first = pairs // (n + 1) if n > 1 else pairs
    return [first] + [(pairs - first) // (n - 1)] * (n - 2) + [pairs - first - (pairs - first) // (n - 1) * (n - 2)] if n > 1 else [first]


# --------------------------------------------------------------------------------------------------------------
# inputs (everything from the seed alone; no package code)
# --------------------------------------------------------------------------------------------------------------

def _gen(seed, *ids):
    g = torch.Generator(device="cuda")
    x = int(seed) & 0x7FFFFFFF
    for i in ids:
        x = (x * 1000003 + int(i) + 17) & 0x7FFFFFFFFFFFFFF
    g.manual_seed(x)
    return g


def _randn(seed, key, shape, kind=torch.float32):
    return torch.randn(shape, generator=_gen(seed, key), device="cuda", dtype=torch.float32).to(kind)


def _kind(case):
    return torch.float16 if case["dtype"] == "f16" else torch.float32


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _cache(case, seed, tokens, layers=1, spare=0):
    """Scattered pages for tokens[b] tokens each: (table, blocks, K pages, V pages)."""
    hk, hd = case["kv_heads"], case["head_dim"]
    need = [-(-t // BLOCK) for t in tokens]
    blocks = sum(need) + spare
    ids = np.random.default_rng(int(seed) & 0x7FFFFFFF).permutation(blocks).astype(np.int32)
    table = np.full((len(tokens), max(max(need), 1)), -1, np.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        at += m
    return (table, blocks, _randn(seed, 3, (layers, blocks, hk, hd // 8, BLOCK, 8), _kind(case)),
            _randn(seed, 4, (layers, blocks, hk, hd, BLOCK), _kind(case)))


def _row_inputs(case, seed):
    n, ks = _shape(case)
    h, hk, hd = case["heads"], case["kv_heads"], case["head_dim"]
    m = sum(ks) + len(ks)
    x = SimpleNamespace(n=n, ks=ks, rows=m)
    x.table, x.blocks, x.k_pages, x.v_pages = _cache(case, seed, [a + k + 1 for a, k in zip(n, ks)])
    qkv = _randn(seed, 1, (m, (h + 2 * hk) * hd), torch.float32 if case["wide"] else _kind(case))
    x.q = qkv[:, :h * hd].view(m, h, hd)
    x.k = qkv[:, h * hd:(h + hk) * hd].view(m, hk, hd)
    x.v = qkv[:, (h + hk) * hd:].view(m, hk, hd)
    x.q_gain, x.k_gain = (1 + 0.1 * _randn(seed, key, (hd,)) if case["norm"] else None for key in (5, 6))
    # axis 0: the token's place in the text; the others: places in pictures of 48 x 48
    place = np.concatenate([np.arange(a, a + k + 1) for a, k in zip(n, ks)])
    x.positions = _i32(np.stack([place, place // 48 % 48, place % 48][:case["axes"]]))
    return x


def _attention_inputs(case, seed):
    n, ks = _shape(case)
    m = sum(ks) + len(ks)
    x = SimpleNamespace(ctx=n, ks=ks, rows=m)
    x.table, x.blocks, x.k, x.v = _cache(case, seed, [a + k + 1 for a, k in zip(n, ks)])
    x.q = _randn(seed, 5, (m, case["heads"], case["head_dim"]), _kind(case))
    return x


def _weigh_inputs(case, seed):
    """Queries, the statistics that their attention left (a reference and the sum of 2^(score - reference)), and the weights so
    far."""
    x = _attention_inputs(case, seed)
    hk, h, hd = case["kv_heads"], case["heads"], case["head_dim"]
    x.n_out = _committed(case)
    x.seen = [a + 3 * b for b, a in enumerate(x.ctx)]
    x.width = x.table.shape[1] * BLOCK
    x.mass = torch.exp(2 * _randn(seed, 7, (1, len(x.ks), hk, x.width)))
    x.born = torch.arange(x.width, dtype=torch.int32, device="cuda").expand(1, len(x.ks), hk, x.width).contiguous()
    x.stats = torch.empty((x.rows, h, 2), device="cuda")
    r = 0
    for b, (c, k) in enumerate(zip(x.ctx, x.ks)):
        keys = _dense(x.k[0], None, _i32(x.table[b]).long(), c + k + 1)[0].float()
        for lo in range(0, k + 1, 1024):
            q = x.q[r + lo:r + min(k + 1, lo + 1024)]
            s = _scores(q, keys, torch.arange(c + lo, c + lo + len(q), device="cuda")) * LOG2E
            top = s.amax(dim=-1)
            x.stats[r + lo:r + lo + len(q), :, 0] = top.permute(1, 0, 2).reshape(len(q), h)
            x.stats[r + lo:r + lo + len(q), :, 1] = torch.exp2(s - top[..., None]).sum(dim=-1).permute(1, 0, 2).reshape(len(q), h)
        r += k + 1
    return x


def _evict_inputs(case, seed):
    n, _ = _shape(case)
    hk, layers = case["kv_heads"], case["layers"]
    x = SimpleNamespace(n=n, slots=len(n))
    x.table, x.blocks, x.k, x.v = _cache(case, seed, n, layers, 8)
    x.width = x.table.shape[1] * BLOCK
    x.held = np.array([-(-t // BLOCK) for t in n], np.int32)
    x.refs = np.zeros(x.blocks, np.int32)
    x.refs[x.table[x.table >= 0]] = 1
    x.mass = torch.exp(2 * _randn(seed, 7, (layers, x.slots, hk, x.width)))
    born = torch.arange(x.width, dtype=torch.int32, device="cuda").expand(layers, x.slots, hk, x.width).clone()
    if case["again"]:
        # every head has lost other tokens: what stands behind the first ones has come from anywhere
        first = case["sinks"]
        for b, t in enumerate(n):
            if t > first:
                order = torch.rand((layers, hk, 2 * (t - first)), generator=_gen(seed, 8, b), device="cuda").argsort(dim=-1)
                born[:, b, :, first:t] = (first + order[..., :t - first]).to(torch.int32)
    x.born = born
    return x


# --------------------------------------------------------------------------------------------------------------
# prepare
# --------------------------------------------------------------------------------------------------------------

def _model(case, layers, max_pos):
    """A library context with the case's head geometry (these entry points read no other parameter)."""
    from paper_2402_15678_amd import harness, synth
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if case["dtype"] == "f16" else synth.DT_F32, layers, 128, case["heads"],
                        case["kv_heads"], case["head_dim"], 128, 8, max_pos)
    return d, harness.DeviceModel.random_on_device(d, 1)


def _prepare_rows(case, seed):
    x = _row_inputs(case, seed)
    s = SimpleNamespace(op="rows", case=case, x=x, table=_i32(x.table), k_pages=x.k_pages, v_pages=x.v_pages,
                        q_out=torch.zeros((x.rows, case["heads"], case["head_dim"]), dtype=_kind(case), device="cuda"))
    if own:
        from paper_2402_15678_amd import harness
        d, s.model = _model(case, 1, x.table.shape[1] * BLOCK)
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, x.n, [x.k_pages[0]], [x.v_pages[0]])
        s.spec = _i32(x.ks)
        s.rule = harness.RowRule(case["rot"], _axis_pairs(case), 10000.0, x.q_gain, x.k_gain, 1e-5)
    else:
        s.slot = torch.cat([torch.arange(a, a + k + 1, device="cuda") for a, k in zip(x.n, x.ks)])
        s.seq = torch.repeat_interleave(torch.arange(len(x.ks), device="cuda"), torch.tensor([k + 1 for k in x.ks], device="cuda"))
    return s


def _prepare_window(case, seed):
    x = _attention_inputs(case, seed)
    s = SimpleNamespace(op="window", case=case, x=x, q=x.q, table=_i32(x.table).long(),
                        out=torch.zeros((x.rows, case["heads"] * case["head_dim"]), dtype=_kind(case), device="cuda"))
    if own:
        from paper_2402_15678_amd import harness
        max_ctx = max(c + k + 1 for c, k in zip(x.ctx, x.ks))
        d, s.model = _model(case, 1, max_ctx)
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, x.ctx, [x.k[0]], [x.v[0]])
        s.spec = _i32(x.ks)
        s.ses = harness.WindowSession(s.model, s.kv, len(x.ks), x.rows, max(x.ks) + 1, max_ctx, case["window"], case["sinks"])
    return s


def _prepare_weigh(case, seed):
    x = _weigh_inputs(case, seed)
    s = SimpleNamespace(op="weigh", case=case, x=x, table=_i32(x.table).long(), mass=x.mass, born=x.born, saved=x.mass.clone())
    if own:
        from paper_2402_15678_amd import harness
        d, s.model = _model(case, 1, x.width)
        # (after the commit the accepted rows are part of the context)
        ctx = [c + a for c, a in zip(x.ctx, x.n_out)] if case["committed"] else x.ctx
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, ctx, [x.k[0]], [x.v[0]])
        s.spec, s.n_out, s.seen = _i32(x.ks), _i32(x.n_out) if case["committed"] else None, _i32(x.seen)
        s.ledger = harness.KVLedger(s.model, s.kv, x.mass, x.born)
    return s


def _prepare_evict(case, seed):
    x = _evict_inputs(case, seed)
    s = SimpleNamespace(op="evict", case=case, x=x, k=x.k, v=x.v, mass=x.mass, born=x.born,
                        saved_mass=x.mass.clone(), saved_born=x.born.clone(), keep=_i32([case["keep"]] * x.slots))
    if own:
        from paper_2402_15678_amd import harness
        d, s.model = _model(case, case["layers"], x.width)
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, x.n, list(s.k), list(s.v))
        s.pool = harness.KVPool(s.model, s.kv, _i32(x.refs), _i32(x.held))
        s.ledger = harness.KVLedger(s.model, s.kv, s.mass, s.born)
        s.saved = s.pool.state.clone()
    else:
        parts = [x.table.reshape(-1), x.refs, x.held, np.array(x.n, np.int32)]
        s.state = _i32(np.concatenate(parts))
        s.saved = s.state.clone()
        s.table, s.refs, s.held, s.ctx = s.state.split([len(p) for p in parts])
        s.table = s.table.view(x.slots, -1)
    return s


def prepare(case, seed):
    return {"rows": _prepare_rows, "window": _prepare_window, "weigh": _prepare_weigh, "evict": _prepare_evict}[case["op"]](case, seed)


# --------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------

def _dense(k, v, ids, n):
    """The first n cached rows behind the blocks `ids`, [Hkv][n][hd] each."""
    ids = ids[:-(-n // BLOCK)]
    k = k[ids]
    k = k.permute(1, 0, 3, 2, 4).reshape(k.shape[1], -1, k.shape[2] * 8)[:, :n]
    if v is None:
        return k, None
    v = v[ids]
    return k, v.permute(1, 0, 3, 2).reshape(v.shape[1], -1, v.shape[2])[:, :n]


def _scores(q, keys, limit):
    """q [rows][H][hd], keys [Hkv][n][hd] in 32 bits, row r sees the keys up to limit[r]: [Hkv][rows][H / Hkv][n]."""
    m, h, hd = q.shape
    hk = keys.shape[0]
    x = q.float().view(m, hk, h // hk, hd).permute(1, 0, 2, 3).reshape(hk, -1, hd) / math.sqrt(hd)
    s = torch.matmul(x, keys.transpose(1, 2).contiguous()).view(hk, m, h // hk, -1)
    hidden = torch.arange(keys.shape[1], device="cuda")[None, :] > limit[:, None]
    return s.masked_fill_(hidden[None, :, None, :], -math.inf)


def _turn(x, gain, case, angle):
    """Norm and rotation of heads [rows][heads][hd] in 32 bits."""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-5) * gain
    half = case["rot"] // 2
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    a, b = x[..., :half], x[..., half:2 * half]
    return torch.cat((a * c - b * s, b * c + a * s, x[..., 2 * half:]), dim=-1)


def _angles(case, positions):
    """[rows][rot / 2] in 64 bits: pair i has its axis' position times 10000^(-2i / rot)."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(_axis_pairs(case), device="cuda"))
    return positions[axis].t().double() * 10000.0 ** (-2 * i / case["rot"])


def _plain_rows(s):
    x, case = s.x, s.case
    angle = _angles(case, x.positions)
    s.q_out.copy_(_turn(x.q, x.q_gain, case, angle))
    k = _turn(x.k, x.k_gain, case, angle).to(s.k_pages.dtype)
    blk, off = s.table[s.seq, s.slot // BLOCK].long(), s.slot % BLOCK
    s.k_pages[0][blk, :, :, off, :] = k.reshape(k.shape[0], k.shape[1], -1, 8)
    s.v_pages[0][blk, :, :, off] = x.v.to(s.v_pages.dtype)
    return {"q": s.q_out, "k_pages": s.k_pages, "v_pages": s.v_pages}


def _own_rows(s):
    from paper_2402_15678_amd import harness
    harness.qk_norm_rope(s.model, s.x.q, s.x.k, s.x.v, s.rule, s.x.positions, s.spec, s.x.ks, s.q_out, kv=s.kv)
    return {"q": s.q_out, "k_pages": s.k_pages, "v_pages": s.v_pages}


def _plain_window(s):
    x, case = s.x, s.case
    h, hk, hd, window, sinks = case["heads"], case["kv_heads"], case["head_dim"], case["window"], case["sinks"]
    r = 0
    for b, (c, k) in enumerate(zip(x.ctx, x.ks)):
        keys, values = (t.float() for t in _dense(x.k[0], x.v[0], s.table[b], c + k + 1))
        step = max(1, min(1024, (1 << 28) // (h * (min(c + k + 1, window + sinks + 1024)))))
        for lo in range(0, k + 1, step):
            q = x.q[r + lo:r + min(k + 1, lo + step)]
            pos = torch.arange(c + lo, c + lo + len(q), device="cuda")
            # the keys that some row sees
            start = max(0, c + lo - window + 1)
            at = torch.cat((torch.arange(min(sinks, start), device="cuda"), torch.arange(start, c + lo + len(q), device="cuda")))
            seen = (at[None, :] <= pos[:, None]) & ((at[None, :] > pos[:, None] - window) | (at[None, :] < sinks))
            z = _scores(q, keys[:, at], torch.full_like(pos, len(at)))
            z.masked_fill_(~seen[None, :, None, :], -math.inf)
            z = torch.exp(z - z.amax(dim=-1, keepdim=True))
            o = torch.matmul(z.view(hk, -1, len(at)), values[:, at]) / z.sum(dim=-1).view(hk, -1, 1)
            s.out[r + lo:r + lo + len(q)] = o.view(hk, len(q), h // hk, hd).permute(1, 0, 2, 3).reshape(len(q), h * hd).to(s.out.dtype)
        r += k + 1
    return s.out


def _own_window(s):
    return s.ses.attention(s.q, s.spec, s.x.ks, s.out)


def _plain_weigh(s):
    x, case = s.x, s.case
    s.mass.copy_(s.saved)
    h, hk = case["heads"], case["kv_heads"]
    r = 0
    for b, (c, k, a) in enumerate(zip(x.ctx, x.ks, x.n_out)):
        n = c + a
        keys = _dense(x.k[0], None, s.table[b], n)[0].float()
        total = torch.zeros((hk, n), device="cuda")
        step = max(1, min(1024, (1 << 28) // (h * n)))
        for lo in range(0, a, step):
            q = x.q[r + lo:r + min(a, lo + step)]
            z = _scores(q, keys, torch.arange(c + lo, c + lo + len(q), device="cuda")) * LOG2E
            st = x.stats[r + lo:r + lo + len(q)].view(len(q), hk, h // hk, 2).permute(1, 0, 2, 3)
            total += (torch.exp2(z - st[..., :1]) / st[..., 1:]).sum(dim=(1, 2))
        total[:, :c] += s.mass[0, b, :, :c]
        s.mass[0, b, :, :n] = total
        s.born[0, b, :, c:n] = x.seen[b] + torch.arange(a, dtype=torch.int32, device="cuda")
        r += k + 1
    return {"mass": s.mass, "born": s.born}


def _own_weigh(s):
    s.mass.copy_(s.saved)
    s.ledger.weigh(s.x.q, s.x.stats, s.spec, s.x.ks, 0, s.x.width, s.n_out, s.seen)
    return {"mass": s.mass, "born": s.born}


def _plain_evict(s):
    x, case = s.x, s.case
    keep = case["keep"]
    for b, n in enumerate(x.n):
        if n <= keep:
            continue
        mass, born = s.mass[:, b, :, :n], s.born[:, b, :, :n]
        always = (born < case["sinks"]) | (born > born.amax(dim=-1, keepdim=True) - case["recent"])
        order = torch.sort(torch.where(always, math.inf, mass), dim=-1, descending=True, stable=True).indices[..., :keep]
        stays = torch.zeros_like(always).scatter_(-1, order, True)
        layer, head, hole = (~stays[..., :keep]).nonzero(as_tuple=True)
        src = stays[..., keep:].nonzero(as_tuple=True)[2] + keep
        row = s.table[b].long()
        to, frm = (row[hole // BLOCK], hole % BLOCK), (row[src // BLOCK], src % BLOCK)
        s.k[layer, to[0], head, :, to[1]] = s.k[layer, frm[0], head, :, frm[1]]
        s.v[layer, to[0], head, :, to[1]] = s.v[layer, frm[0], head, :, frm[1]]
        mass[layer, head, hole] = mass[layer, head, src]
        born[layer, head, hole] = born[layer, head, src]
        held = -(-keep // BLOCK)
        gone = s.table[b, held:x.held[b]].long()
        s.refs[gone] -= 1
        s.table[b, held:x.held[b]] = -1
        s.held[b] = held
        s.ctx[b] = keep


def _run_evict(s):
    # (the mapping, the weights and the order as they were before the pass; what is evicted goes to the same places again)
    s.mass.copy_(s.saved_mass)
    s.born.copy_(s.saved_born)
    if own:
        s.pool.state.copy_(s.saved)
        s.pool.evict(s.keep, s.case["sinks"], s.case["recent"], s.ledger)
        return {"table": s.kv.block_tables, "refs": s.pool.block_refs, "held": s.pool.seq_blocks, "ctx": s.kv.ctx_lens,
                "k": s.k, "v": s.v, "mass": s.mass, "born": s.born}
    s.state.copy_(s.saved)
    _plain_evict(s)
    return {"table": s.table, "refs": s.refs, "held": s.held, "ctx": s.ctx, "k": s.k, "v": s.v, "mass": s.mass, "born": s.born}


def run(state):
    if state.op == "evict":
        return _run_evict(state)
    if state.op == "rows":
        return _own_rows(state) if own else _plain_rows(state)
    if state.op == "window":
        return _own_window(state) if own else _plain_window(state)
    return _own_weigh(state) if own else _plain_weigh(state)


# --------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------------

def _visible(c, k, window, sinks):
    """(keys that some row of the sequence sees, pairs of a row and a key that it sees)."""
    pos = np.arange(c, c + k + 1, dtype=np.int64)
    start = np.maximum(0, pos - window + 1)
    first = int(start[0])
    return c + k + 1 - first + min(sinks, first), int((pos + 1 - start + np.minimum(sinks, start)).sum())


def work(case):
    n, ks = _shape(case)
    es = 2.0 if case["dtype"] == "f16" else 4.0
    h, hk, hd = case["heads"], case["kv_heads"], case["head_dim"]
    rows = sum(ks) + len(ks)
    if case["op"] == "rows":
        heads = h + 2 * hk
        return {"bytes": rows * heads * hd * ((4.0 if case["wide"] else es) + es) + 4.0 * rows * case["axes"],
                "flops": rows * hd * (h + hk) * (7.0 if case["norm"] else 3.0)}
    if case["op"] == "window":
        seen = [_visible(c, k, case["window"], case["sinks"]) for c, k in zip(n, ks)]
        return {"bytes": (sum(a for a, _ in seen) * 2 * hk + rows * 2 * h) * hd * es, "flops": 4.0 * h * hd * sum(p for _, p in seen)}
    if case["op"] == "weigh":
        out = _committed(case)
        keys = sum(c + a for c, a in zip(n, out))
        pairs = sum(a * c + a * (a + 1) // 2 for c, a in zip(n, out))
        return {"bytes": keys * hk * (hd * es + 4.0) + sum(n) * hk * 4.0 + sum(out) * (h * (hd * es + 8.0) + hk * 4.0),
                "flops": 2.0 * h * hd * pairs}
    # (how many tokens change places depends on the weights: the expected number, were they alike)
    keep = case["keep"]
    cut = [t for t in n if t > keep]
    moved = sum(keep * (1.0 - keep / t) for t in cut)
    per = case["layers"] * hk
    ints = sum(per * t * 8.0 for t in cut) + 16.0 * sum(-(-t // BLOCK) for t in cut) + 8.0 * len(n)
    return {"bytes": per * moved * 2.0 * (2 * hd * es + 8.0) + ints, "flops": 0.0}


# --------------------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------------------

def _exact_rows(case, seed):
    x = _row_inputs(case, seed)
    half = case["rot"] // 2
    axis_of = [a for a, p in enumerate(_axis_pairs(case)) for _ in range(p)]
    freq = torch.tensor([10000.0 ** (-2.0 * i / case["rot"]) for i in range(half)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones_like(freq).expand(x.rows, half), x.positions.double()[axis_of].transpose(0, 1) * freq)

    def heads(t, gain):
        t = t.double()
        if gain is not None:
            t = t / torch.sqrt(t.pow(2).sum(dim=2, keepdim=True) / t.shape[2] + 1e-5) * gain.double()
        z = torch.complex(t[:, :, :half].contiguous(), t[:, :, half:2 * half].contiguous()) * turn[:, None]
        return torch.cat((z.real, z.imag, t[:, :, 2 * half:]), dim=2)

    q, k = heads(x.q, x.q_gain), heads(x.k, x.k_gain)
    kp, vp = x.k_pages.double(), x.v_pages.double()
    r = 0
    for b, (c, m) in enumerate(zip(x.n, x.ks)):
        at = c
        while at < c + m + 1:
            blk, off = int(x.table[b, at // BLOCK]), at % BLOCK
            w = min(BLOCK - off, c + m + 1 - at)
            rows = slice(r + at - c, r + at - c + w)
            kp[0, blk, :, :, off:off + w, :] = k[rows].view(w, case["kv_heads"], -1, 8).permute(1, 2, 0, 3)
            vp[0, blk, :, :, off:off + w] = x.v[rows].double().permute(1, 2, 0)
            at += w
        r += m + 1
    return {"q": q, "k_pages": kp, "v_pages": vp}


def _sequence(x, b, n):
    """The first n cached rows of sequence b, [n][Hkv][hd] each."""
    ids = torch.from_numpy(x.table[b, :-(-n // BLOCK)].astype(np.int64)).cuda()
    k, v = x.k[0][ids], x.v[0][ids]
    return (k.permute(0, 3, 1, 2, 4).reshape(-1, k.shape[1], k.shape[2] * 8)[:n], v.permute(0, 3, 1, 2).reshape(-1, v.shape[1], v.shape[2])[:n])


def _exact_window(case, seed):
    x = _attention_inputs(case, seed)
    h, hk, hd, window, sinks = case["heads"], case["kv_heads"], case["head_dim"], case["window"], case["sinks"]
    out = torch.empty((x.rows, h, hd), dtype=torch.float64, device="cuda")
    r = 0
    for b, (c, m) in enumerate(zip(x.ctx, x.ks)):
        k, v = _sequence(x, b, c + m + 1)
        for lo in range(0, m + 1, 2048):
            hi = min(m + 1, lo + 2048)
            first = max(0, c + lo - window + 1)
            edge = min(sinks, first)
            pos = torch.arange(c + lo, c + hi, device="cuda")[:, None]
            key = torch.cat((torch.arange(edge, device="cuda"), torch.arange(first, c + hi, device="cuda")))[None, :]
            hidden = (key > pos) | ((key <= pos - window) & (key >= sinks))
            for head in range(h):
                kh, vh = (torch.cat((t[:edge, head // (h // hk)], t[first:c + hi, head // (h // hk)])).double() for t in (k, v))
                score = torch.mm(x.q[r + lo:r + hi, head].double(), kh.t().contiguous()) * (hd ** -0.5)
                out[r + lo:r + hi, head] = torch.mm(torch.softmax(score.masked_fill(hidden, -math.inf), dim=1), vh)
        r += m + 1
    return out.reshape(x.rows, h * hd)


def _exact_weigh(case, seed):
    x = _weigh_inputs(case, seed)
    h, hk, hd = case["heads"], case["kv_heads"], case["head_dim"]
    mass, born = x.mass.double(), x.born.clone()
    r = 0
    for b, (c, m, a) in enumerate(zip(x.ctx, x.ks, x.n_out)):
        k, _ = _sequence(x, b, c + a)
        mass[0, b, :, c:c + a] = 0
        born[0, b, :, c:c + a] = torch.arange(x.seen[b], x.seen[b] + a, device="cuda")
        key = torch.arange(c + a, device="cuda")[None, :]
        for head in range(h):
            g = head // (h // hk)
            kt = k[:, g].double().t().contiguous()
            for lo in range(0, a, 2048):
                hi = min(a, lo + 2048)
                z = torch.mm(x.q[r + lo:r + hi, head].double(), kt) * (hd ** -0.5)
                st = x.stats[r + lo:r + hi, head].double()
                p = torch.exp(z - st[:, :1] * math.log(2.0)) / st[:, 1:]
                mass[0, b, g, :c + a] += p.masked_fill(key > torch.arange(c + lo, c + hi, device="cuda")[:, None], 0.0).sum(dim=0)
        r += m + 1
    return {"mass": mass, "born": born}


def _exact_evict(case, seed):
    """One head of one layer of one sequence at a time, with lists."""
    x = _evict_inputs(case, seed)
    keep, hk = case["keep"], case["kv_heads"]
    table, refs, held, ctx = x.table.copy(), x.refs.copy(), x.held.copy(), list(x.n)
    k, v = x.k.double(), x.v.double()
    mass, born = x.mass.cpu().numpy().copy(), x.born.cpu().numpy().copy()
    for b, n in enumerate(x.n):
        if n <= keep:
            continue
        moves = []
        for layer in range(case["layers"]):
            for head in range(hk):
                m, o = mass[layer, b, head, :n], born[layer, b, head, :n]
                last = int(o.max())
                value = np.where((o < case["sinks"]) | (o > last - case["recent"]), np.inf, m)
                chosen = set(np.lexsort((np.arange(n), -value))[:keep].tolist())
                holes = [i for i in range(keep) if i not in chosen]
                movers = [i for i in range(keep, n) if i in chosen]
                m[holes], o[holes] = m[movers], o[movers]
                moves += [(layer, head, i, j) for i, j in zip(holes, movers)]
        if moves:
            layer, head, to, frm = np.array(moves, np.int64).T
            at = lambda slot: (table[b, slot // BLOCK].astype(np.int64), slot % BLOCK)  # noqa: E731
            dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
            (tb, to), (fb, fo) = at(to), at(frm)
            for pages in (k, v):
                idx = (dev(layer), dev(tb), dev(head)), (dev(layer), dev(fb), dev(head))
                pages[idx[0][0], idx[0][1], idx[0][2], :, dev(to)] = pages[idx[1][0], idx[1][1], idx[1][2], :, dev(fo)]
        now = -(-keep // BLOCK)
        refs[table[b, now:held[b]]] -= 1
        table[b, now:held[b]] = -1
        held[b], ctx[b] = now, keep
    return {"table": _i32(table), "refs": _i32(refs), "held": _i32(held), "ctx": _i32(ctx), "k": k, "v": v,
            "mass": torch.from_numpy(mass).cuda().double(), "born": torch.from_numpy(born).cuda()}


def exact(case, seed):
    return {"rows": _exact_rows, "window": _exact_window, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](case, seed)
