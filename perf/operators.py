"""What the operators around a shared paged cache cost: attention over whole prompts, attention of a batch that shares a
long prefix, and the pool of cache pages behind both.

A serving program meets them in this order: a prompt's rows attend to one another and enter the cache (``prompt``), the
request is forked into several that share its pages and get room for their next tokens (``pages``, branch), every step's
attention then reads the shared pages once for all of them (``prefix``), and requests that are done give their blocks back
and the pool is packed together (``pages``, retire).

``own`` false: plain torch, 32 bits.  ``own`` true: the library's entry points.  Head geometries are those of the
repository's model descriptions (64/8 x 128, 40 x 128, 12 x 64 in 16 bits, 4 x 64 in 32) and a few generic ones; cached
rows are N(0, 1), pages are scattered at random over the pool.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

BLOCK = 16
H70B, H13B, HSSM, HTINY = (64, 8, 128, "f16"), (40, 40, 128, "f16"), (12, 12, 64, "f16"), (4, 4, 64, "f32")
GEOMETRIES = (H70B, H70B, H13B, H13B, HSSM, HTINY, (32, 4, 128, "f16"), (16, 2, 64, "f16"), (8, 8, 32, "f16"),
              (8, 2, 256, "f16"), (8, 2, 128, "f32"))


# --------------------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------------------

def _geometry(g):
    return {"heads": g[0], "kv_heads": g[1], "head_dim": g[2], "dtype": g[3]}


def _prompt(g, batch, lo, hi, cache, shape_seed):
    return dict(_geometry(g), op="prompt", batch=batch, lo=lo, hi=hi, cache=cache, shape_seed=shape_seed)


def _prefix(g, batch, prefix, lo, hi, k_lo, k_hi, shape_seed):
    """`lo` .. `hi`: cached tokens of a sequence behind the prefix; `k_lo` .. `k_hi`: speculated tokens."""
    return dict(_geometry(g), op="prefix", batch=batch, prefix=prefix, lo=lo, hi=hi, k_lo=k_lo, k_hi=k_hi, shape_seed=shape_seed)


def _branch(g, layers, batch, children, lo, hi, room, shape_seed):
    return dict(_geometry(g), op="pages", kind="branch", layers=layers, batch=batch, children=children, lo=lo, hi=hi, room=room,
                shape_seed=shape_seed)


def _retire(g, layers, batch, gone, lo, hi, shape_seed):
    return dict(_geometry(g), op="pages", kind="retire", layers=layers, batch=batch, gone=gone, lo=lo, hi=hi, shape_seed=shape_seed)


def listed():
    named = lambda name, c: dict(c, name=name)  # noqa: E731
    return [
        # the smallest prompt: one short request on a drafting model, where launch and latency count
        named("prompt-ssm-b1-len37", _prompt(HSSM, 1, 37, 37, False, 1)),
        # a small fp32 model, ragged prompts, rows written into the cache as well
        named("prompt-tiny-fp32-b4-cache", _prompt(HTINY, 4, 33, 700, True, 2)),
        # a mid-size model without head groups: a batch of ragged prompts entering the cache
        named("prompt-13b-b8-ragged-cache", _prompt(H13B, 8, 60, 1500, True, 3)),
        # the large model's long prompts: bound by the matrix cores
        named("prompt-70b-b3-long", _prompt(H70B, 3, 3000, 7000, False, 4)),
        # the smallest step on a shared prompt: three branches of one short request, fp32
        named("prefix-tiny-fp32-b3-p48-k4", _prefix(HTINY, 3, 48, 0, 30, 4, 4, 5)),
        # one token each for 16 requests behind a common instruction, no head groups
        named("prefix-13b-b16-p1024-decode", _prefix(H13B, 16, 1024, 0, 600, 0, 0, 6)),
        # a full server behind one long document, 8 speculated tokens each
        named("prefix-70b-b64-p8192-k8", _prefix(H70B, 64, 8192, 16, 400, 8, 8, 7)),
        # few rows, very long prefix: a stream of keys
        named("prefix-70b-b3-p32000-decode", _prefix(H70B, 3, 32000, 0, 300, 0, 2, 8)),
        # one request becomes four on a small model: bookkeeping and latency
        named("pages-branch-tiny-b1x4", _branch(HTINY, 2, 1, 4, 100, 100, 5, 9)),
        # 16 requests become four each, every branch with room for its next 9 tokens
        named("pages-branch-70b-b16x4", _branch(H70B, 8, 16, 4, 100, 700, 9, 10)),
        # a drafting model's pool after a third of its requests have finished
        named("pages-retire-ssm-b48", _retire(HSSM, 12, 48, 16, 50, 900, 11)),
        # a large pool, half of the requests gone: half of the blocks move
        named("pages-retire-70b-b24", _retire(H70B, 8, 24, 12, 200, 800, 12)),
    ]


def _log_int(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    g = rng.choice(GEOMETRIES)
    seed = rng.randrange(1 << 20)
    span = lambda lo, hi: sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))  # noqa: E731
    pick = rng.randrange(3)
    if pick == 0:
        batch = _log_int(rng, 1, 24)
        most = int(math.sqrt(8e7 * 64 * 128 / (batch * g[0] * g[2]) / (4 if g[3] == "f32" or g[2] not in (64, 128) else 1)))
        return _prompt(g, batch, *span(1, max(2, min(most, 7000 if batch < 4 else 2500))), rng.random() < 0.5, seed)
    if pick == 1:
        batch = _log_int(rng, 1, 64)
        k_hi = rng.choice((0, rng.randint(0, 12)))
        k_lo = rng.randint(0, k_hi)
        most = 8192 * 64 * 9 * 64 * 128 // (batch * (k_hi + 1) * g[0] * g[2]) // (4 if g[3] == "f32" or g[2] not in (64, 128) else 1)
        prefix = BLOCK * _log_int(rng, 1, max(2, min(most, 32000) // BLOCK))
        lo, hi = span(1, 600)
        return _prefix(g, batch, prefix, lo - 1, hi, k_lo, k_hi, seed)
    layers = rng.randint(1, 8)
    if rng.random() < 0.5:
        return _branch(g, layers, _log_int(rng, 1, 16), rng.randint(1, 4), *span(1, 700), rng.randint(1, 17), seed)
    batch = _log_int(rng, 2, 32)
    return _retire(g, layers, batch, rng.randint(1, batch), *span(16, 700), seed)


def _shape(case):
    """Lengths of the batch, from the case alone."""
    r = random.Random(case["shape_seed"])
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    ks = [r.randint(case["k_lo"], case["k_hi"]) for _ in range(case["batch"])] if case["op"] == "prefix" else None
    return n, ks


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


def _randn(seed, key, shape, kind):
    return torch.randn(shape, generator=_gen(seed, key), device="cuda", dtype=torch.float32).to(kind)


def _kind(case):
    return torch.float16 if case["dtype"] == "f16" else torch.float32


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _pages(case, layers, blocks, seed, zero=False):
    hk, hd = case["kv_heads"], case["head_dim"]
    ks, vs = (layers, blocks, hk, hd // 8, BLOCK, 8), (layers, blocks, hk, hd, BLOCK)
    if zero:
        return torch.zeros(ks, dtype=_kind(case), device="cuda"), torch.zeros(vs, dtype=_kind(case), device="cuda")
    return _randn(seed, 3, ks, _kind(case)), _randn(seed, 4, vs, _kind(case))


def _ids(seed, count, pool=None):
    """`count` block ids in random order, out of a pool of that many (or more)."""
    return np.random.default_rng(int(seed) & 0x7FFFFFFF).permutation(pool or count)[:count].astype(np.int32)


def _prompt_inputs(case, seed):
    """The rows of a fused projection (queries, keys, values side by side) and the places in the cache."""
    n, _ = _shape(case)
    h, hk, hd = case["heads"], case["kv_heads"], case["head_dim"]
    row0 = np.concatenate(([0], np.cumsum(n))).astype(np.int32)
    qkv = _randn(seed, 1, (int(row0[-1]), (h + 2 * hk) * hd), _kind(case))
    need = [-(-x // BLOCK) for x in n]
    table = np.full((len(n), max(need)), -1, np.int32)
    ids = _ids(seed, sum(need))
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        at += m
    x = SimpleNamespace(n=n, row0=row0, qkv=qkv, table=table, blocks=sum(need))
    x.q = qkv[:, :h * hd].view(-1, h, hd)
    x.k = qkv[:, h * hd:(h + hk) * hd].view(-1, hk, hd)
    x.v = qkv[:, (h + hk) * hd:].view(-1, hk, hd)
    return x


def _prefix_inputs(case, seed):
    n, ks = _shape(case)
    p = case["prefix"] // BLOCK
    need = [-(-(x + k + 1) // BLOCK) for x, k in zip(n, ks)]
    ids = _ids(seed, p + sum(need))
    table = np.full((len(n), p + max(need)), -1, np.int32)
    table[:, :p] = ids[:p]
    at = p
    for b, m in enumerate(need):
        table[b, p:p + m] = ids[at:at + m]
        at += m
    k, v = _pages(case, 1, len(ids), seed)
    rows = sum(ks) + len(ks)
    q = _randn(seed, 5, (rows, case["heads"], case["head_dim"]), _kind(case))
    return SimpleNamespace(ctx=[case["prefix"] + x for x in n], ks=ks, table=table, blocks=len(ids), k=k, v=v, q=q, rows=rows)


def _pool_inputs(case, seed):
    """Sequences in the first slots, their blocks scattered over the pool; branch: empty slots behind them for the children,
    a share of free blocks; retire: the pool is nearly full."""
    n, _ = _shape(case)
    need = [-(-x // BLOCK) for x in n]
    live = sum(need)
    if case["kind"] == "branch":
        slots = len(n) * (1 + case["children"])
        spare = slots * (2 + -(-case["room"] // BLOCK))
        width = max(need) + 2 + case["room"] // BLOCK
    else:
        slots, spare, width = len(n), 8, max(need)
    blocks = live + spare
    ids = _ids(seed, live, blocks)
    state = SimpleNamespace(table=np.full((slots, width), -1, np.int32), refs=np.zeros(blocks, np.int32),
                            held=np.zeros(slots, np.int32), ctx=np.zeros(slots, np.int32), slots=slots, width=width, blocks=blocks)
    at = 0
    for b, m in enumerate(need):
        state.table[b, :m] = ids[at:at + m]
        at += m
        state.held[b], state.ctx[b] = m, n[b]
    state.refs[ids] = 1
    if case["kind"] == "branch":
        state.src = np.repeat(np.arange(len(n), dtype=np.int32), case["children"])
        state.dst = np.arange(len(n), slots, dtype=np.int32)
        state.tokens = (np.concatenate((state.ctx[:len(n)], state.ctx[state.src])) + case["room"]).astype(np.int32)
    else:
        r = random.Random(case["shape_seed"] + 1)
        state.gone = np.array(sorted(r.sample(range(len(n)), case["gone"])), np.int32)
    return state


# --------------------------------------------------------------------------------------------------------------
# prepare
# --------------------------------------------------------------------------------------------------------------

def _model(case, layers, max_pos):
    """A library context with the case's head geometry (these entry points read no other parameter)."""
    from paper_2402_15678_amd import harness, synth
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if case["dtype"] == "f16" else synth.DT_F32, layers, 128, case["heads"],
                        case["kv_heads"], case["head_dim"], 128, 8, max_pos)
    return d, harness.DeviceModel.random_on_device(d, 1)


def _prepare_prompt(case, seed):
    x = _prompt_inputs(case, seed)
    s = SimpleNamespace(op="prompt", case=case, q=x.q, k=x.k, v=x.v, n=x.n, h_row0=x.row0.tolist(), row0=_i32(x.row0),
                        out=torch.zeros((len(x.qkv), case["heads"] * case["head_dim"]), dtype=_kind(case), device="cuda"))
    if case["cache"]:
        s.k_pages, s.v_pages = _pages(case, 1, x.blocks, seed, zero=True)
        s.table = _i32(x.table)
    if own:
        from paper_2402_15678_amd import harness
        d, s.model = _model(case, 1, max(x.n))
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, [0] * len(x.n), [s.k_pages[0]], [s.v_pages[0]]) if case["cache"] else None
        s.plan = harness.PromptRows(s.h_row0)
    return s


def _prepare_prefix(case, seed):
    x = _prefix_inputs(case, seed)
    s = SimpleNamespace(op="prefix", case=case, q=x.q, k=x.k, v=x.v, ctx=x.ctx, ks=x.ks, table=_i32(x.table), spec=_i32(x.ks),
                        out=torch.zeros((x.rows, case["heads"] * case["head_dim"]), dtype=_kind(case), device="cuda"))
    if own:
        from paper_2402_15678_amd import harness
        max_ctx = max(c + k + 1 for c, k in zip(x.ctx, x.ks))
        d, s.model = _model(case, 1, max_ctx)
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, x.ctx, [x.k[0]], [x.v[0]])
        s.ses = harness.PrefixSession(s.model, s.kv, len(x.ks), x.rows, case["prefix"], max_ctx)
    return s


def _prepare_pages(case, seed):
    x = _pool_inputs(case, seed)
    s = SimpleNamespace(op="pages", case=case, x=x)
    s.k, s.v = _pages(case, case["layers"], x.blocks, seed)
    lists = ("src", "dst", "tokens") if case["kind"] == "branch" else ("gone",)
    for key in lists:
        setattr(s, key, _i32(getattr(x, key)))
    if own:
        from paper_2402_15678_amd import harness
        d, s.model = _model(case, case["layers"], x.width * BLOCK)
        s.kv = harness.DeviceKV(d, BLOCK, x.blocks, x.table, x.ctx, list(s.k), list(s.v))
        s.pool = harness.KVPool(s.model, s.kv, _i32(x.refs), _i32(x.held))
        s.saved = s.pool.state.clone()
    else:
        parts = [x.table.reshape(-1), x.refs, x.held, x.ctx]
        s.state = _i32(np.concatenate(parts))
        s.saved = s.state.clone()
        cut = np.cumsum([len(p) for p in parts])
        s.table, s.refs, s.held, s.ctx = (s.state[a:b] for a, b in zip([0, *cut[:-1]], cut))
        s.table = s.table.view(x.slots, x.width)
    return s


def prepare(case, seed):
    return {"prompt": _prepare_prompt, "prefix": _prepare_prefix, "pages": _prepare_pages}[case["op"]](case, seed)


# --------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------

def _attend(q, k, v, limit, out):
    """q [rows][H][hd], k and v [Hkv][keys][hd] in 32 bits; row r sees the keys up to limit[r]; result into out [rows][H * hd]."""
    rows, h, hd = q.shape
    hk = k.shape[0]
    kt = k.transpose(1, 2).contiguous()
    step = max(1, (1 << 28) // (h * k.shape[1]))
    at = torch.arange(k.shape[1], device="cuda")
    for r in range(0, rows, step):
        x = q[r:r + step]
        m = len(x)
        x = x.float().view(m, hk, h // hk, hd).permute(1, 0, 2, 3).reshape(hk, m * (h // hk), hd) / math.sqrt(hd)
        s = torch.matmul(x, kt).view(hk, m, h // hk, -1)
        s.masked_fill_((at[None, :] > limit[r:r + step, None])[None, :, None, :], -math.inf)
        s = torch.exp(s - s.amax(dim=-1, keepdim=True))
        o = torch.matmul(s.view(hk, m * (h // hk), -1), v) / s.sum(dim=-1).view(hk, -1, 1)
        out[r:r + step] = o.view(hk, m, h // hk, hd).permute(1, 0, 2, 3).reshape(m, h * hd).to(out.dtype)


def _plain_prompt(s):
    for b, n in enumerate(s.n):
        r = slice(s.h_row0[b], s.h_row0[b + 1])
        k, v = s.k[r].float().transpose(0, 1).contiguous(), s.v[r].float().transpose(0, 1).contiguous()
        _attend(s.q[r], k, v, torch.arange(n, device="cuda"), s.out[r])
    got = {"out": s.out}
    if s.case["cache"]:
        at = torch.cat([torch.arange(n, device="cuda") for n in s.n])
        seq = torch.repeat_interleave(torch.arange(len(s.n), device="cuda"), torch.tensor(s.n, device="cuda"))
        blk, off = s.table[seq, at // BLOCK].long(), at % BLOCK
        s.k_pages[0][blk, :, :, off, :] = s.k.reshape(s.k.shape[0], s.k.shape[1], -1, 8)
        s.v_pages[0][blk, :, :, off] = s.v
        got.update(k_pages=s.k_pages, v_pages=s.v_pages)
    return got


def _own_prompt(s):
    from paper_2402_15678_amd import harness
    harness.prompt_attention(s.model, s.q, s.k, s.v, s.row0, s.plan, s.out, s.kv)
    return {"out": s.out, "k_pages": s.k_pages, "v_pages": s.v_pages} if s.case["cache"] else {"out": s.out}


def _rows_of(k, v, ids, n):
    """The first n cached rows behind the blocks `ids`, [Hkv][n][hd] each."""
    k, v = k[ids], v[ids]
    hk, hd = v.shape[1], v.shape[2]
    return (k.permute(1, 0, 3, 2, 4).reshape(hk, -1, hd)[:, :n], v.permute(1, 0, 3, 2).reshape(hk, -1, hd)[:, :n])


def _plain_prefix(s):
    p = s.case["prefix"]
    pk, pv = (t.float() for t in _rows_of(s.k[0], s.v[0], s.table[0, :p // BLOCK].long(), p))
    r = 0
    for b, (c, k) in enumerate(zip(s.ctx, s.ks)):
        n = c - p + k + 1
        ids = s.table[b, p // BLOCK:p // BLOCK - (-n // BLOCK)].long()
        sk, sv = (t.float() for t in _rows_of(s.k[0], s.v[0], ids, n))
        _attend(s.q[r:r + k + 1], torch.cat((pk, sk), dim=1), torch.cat((pv, sv), dim=1),
                torch.arange(c, c + k + 1, device="cuda"), s.out[r:r + k + 1])
        r += k + 1
    return s.out


def _own_prefix(s):
    return s.ses.attention(s.q, s.spec, s.ks, s.out)


def _plain_fork(s, src, dst):
    """The children hold the blocks of their parents' tokens."""
    nb = (s.ctx[src] + BLOCK - 1) // BLOCK
    at = torch.arange(s.table.shape[1], device="cuda")[None, :]
    shared = at < nb[:, None]
    rows = s.table[src]
    s.table[dst] = torch.where(shared, rows, s.table[dst])
    s.refs.index_add_(0, rows[shared].long(), torch.ones_like(rows[shared]))
    s.held[dst] = nb
    s.ctx[dst] = s.ctx[src]


def _plain_reserve(s, tokens):
    """Every sequence may write up to `tokens`: missing blocks are added, shared ones that would be written are replaced."""
    b = len(tokens)
    table = s.table[:b]
    first, need = s.ctx[:b] // BLOCK, (tokens + BLOCK - 1) // BLOCK
    at = torch.arange(table.shape[1], device="cuda")[None, :]
    inside = (at >= first[:, None]) & (at < need[:, None])
    mapped = at < s.held[:b, None]
    shared = inside & mapped & (s.refs[table.clamp(min=0).long()] > 1)
    fresh = shared | (inside & ~mapped)
    free = (s.refs == 0).nonzero().view(-1)
    count = int(fresh.sum())
    given = free[:count]
    old = table[fresh].long()
    part = (shared & (at == first[:, None]) & (s.ctx[:b, None] % BLOCK != 0))[fresh]
    was_shared = shared[fresh]
    s.k[:, given[part]] = s.k[:, old[part]]
    s.v[:, given[part]] = s.v[:, old[part]]
    s.refs.index_add_(0, old[was_shared], torch.full_like(old[was_shared], -1, dtype=torch.int32))
    s.refs[given] = 1
    table[fresh] = given.to(torch.int32)
    s.held[:b] = torch.maximum(s.held[:b], need)


def _plain_free(s, gone):
    rows = s.table[gone]
    held = torch.arange(rows.shape[1], device="cuda")[None, :] < s.held[gone][:, None]
    s.refs.index_add_(0, rows[held].long(), torch.full_like(rows[held], -1))
    s.table[gone] = torch.where(held, torch.full_like(rows, -1), rows)
    s.held[gone] = 0
    s.ctx[gone] = 0


def _plain_compact(s):
    live = s.refs > 0
    n = live.sum()
    at = torch.arange(len(s.refs), device="cuda")
    src, dst = (live & (at >= n)).nonzero().view(-1), (~live & (at < n)).nonzero().view(-1)
    s.k[:, dst] = s.k[:, src]
    s.v[:, dst] = s.v[:, src]
    s.refs[dst] = s.refs[src]
    s.refs[src] = 0
    move = at.to(torch.int32)
    move[src] = dst.to(torch.int32)
    held = torch.arange(s.table.shape[1], device="cuda")[None, :] < s.held[:, None]
    s.table.copy_(torch.where(held, move[s.table.clamp(min=0).long()], s.table))
    return n.to(torch.int32).view(1)


def _run_pages(s):
    # (the mapping as it was before the pass, in one copy)
    if own:
        s.pool.state.copy_(s.saved)
        if s.case["kind"] == "branch":
            s.pool.fork(s.src, s.dst)
            s.pool.reserve(s.tokens)
        else:
            s.pool.free(s.gone)
            s.pool.compact()
        got = {"table": s.kv.block_tables, "refs": s.pool.block_refs, "held": s.pool.seq_blocks, "ctx": s.kv.ctx_lens, "k": s.k, "v": s.v}
        if s.case["kind"] == "retire":
            got["live"] = s.pool.n_live
        return got
    s.state.copy_(s.saved)
    got = {"table": s.table, "refs": s.refs, "held": s.held, "ctx": s.ctx, "k": s.k, "v": s.v}
    if s.case["kind"] == "branch":
        _plain_fork(s, s.src.long(), s.dst.long())
        _plain_reserve(s, s.tokens)
    else:
        _plain_free(s, s.gone.long())
        got["live"] = _plain_compact(s)
    return got


def run(state):
    if state.op == "pages":
        return _run_pages(state)
    if state.op == "prompt":
        return _own_prompt(state) if own else _plain_prompt(state)
    return _own_prefix(state) if own else _plain_prefix(state)


# --------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------------

def work(case):
    n, ks = _shape(case)
    es = 2.0 if case["dtype"] == "f16" else 4.0
    h, hk, hd = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "prompt":
        rows = sum(n)
        return {"bytes": rows * (2 * h + 2 * hk + (2 * hk if case["cache"] else 0)) * hd * es,
                "flops": 4.0 * h * hd * sum(x * (x + 1) // 2 for x in n)}
    if case["op"] == "prefix":
        rows, p = sum(ks) + len(ks), case["prefix"]
        keys = p + sum(x + k + 1 for x, k in zip(n, ks))
        pairs = sum((k + 1) * (p + x) + (k + 1) * (k + 2) // 2 for x, k in zip(n, ks))
        return {"bytes": (keys * 2 * hk + rows * 2 * h) * hd * es, "flops": 4.0 * h * hd * pairs}
    x = _pool_inputs(case, 0)
    if case["kind"] == "branch":
        part = [t % BLOCK != 0 for t in n]
        moved = sum(1 + case["children"] for t in part if t)
    else:
        # (which blocks are live and beyond the packed range depends on the seed: the expected number)
        held = x.held.sum() - x.held[x.gone].sum()
        moved = held * (1.0 - held / x.blocks)
    ints = 2.0 * 4 * (x.refs.size + x.held.size + x.ctx.size + int(x.held.sum()))
    return {"bytes": 2.0 * moved * case["layers"] * 2 * hk * hd * BLOCK * es + ints, "flops": 0.0}


# --------------------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------------------

def _softmax_rows(case, q, k, v, first):
    """Query row i at position first + i; one KV head after the other."""
    h, hk = case["heads"], case["kv_heads"]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    pos = torch.arange(first, first + len(q), device="cuda")
    key = torch.arange(len(k), device="cuda")
    step = max(1, (1 << 27) // len(k))
    for head in range(h):
        kh, vh = k[:, head // (h // hk)].double(), v[:, head // (h // hk)].double()
        for r in range(0, len(q), step):
            last = min(len(k), first + r + step)
            score = torch.mm(q[r:r + step, head].double(), kh[:last].t().contiguous()) * (case["head_dim"] ** -0.5)
            score = score.masked_fill(key[None, :last] > pos[r:r + step, None], -math.inf)
            out[r:r + step, head] = torch.mm(torch.softmax(score, dim=1), vh[:last])
    return out.reshape(len(q), -1)


def _exact_prompt(case, seed):
    x = _prompt_inputs(case, seed)
    parts = [slice(int(a), int(b)) for a, b in zip(x.row0[:-1], x.row0[1:])]
    got = {"out": torch.cat([_softmax_rows(case, x.q[r], x.k[r], x.v[r], 0) for r in parts])}
    if case["cache"]:
        kp, vp = (t.double() for t in _pages(case, 1, x.blocks, seed, zero=True))
        for b, r in enumerate(parts):
            for i, blk in enumerate(x.table[b]):
                m = min(BLOCK, x.n[b] - i * BLOCK)
                if m <= 0:
                    break
                kr, vr = x.k[r][i * BLOCK:i * BLOCK + m].double(), x.v[r][i * BLOCK:i * BLOCK + m].double()
                kp[0, int(blk), :, :, :m, :] = kr.view(m, case["kv_heads"], -1, 8).permute(1, 2, 0, 3)
                vp[0, int(blk), :, :, :m] = vr.permute(1, 2, 0)
        got.update(k_pages=kp, v_pages=vp)
    return got


def _exact_prefix(case, seed):
    x = _prefix_inputs(case, seed)
    outs, r = [], 0
    hk, hd = case["kv_heads"], case["head_dim"]
    for b, (c, m) in enumerate(zip(x.ctx, x.ks)):
        n = c + m + 1
        ids = torch.from_numpy(x.table[b, :-(-n // BLOCK)].astype(np.int64)).cuda()
        k = x.k[0][ids].permute(0, 3, 1, 2, 4).reshape(-1, hk, hd)[:n]
        v = x.v[0][ids].permute(0, 3, 1, 2).reshape(-1, hk, hd)[:n]
        outs.append(_softmax_rows(case, x.q[r:r + m + 1], k, v, c))
        r += m + 1
    return torch.cat(outs)


def _exact_pages(case, seed):
    """The pool as lists and counts, one block at a time."""
    x = _pool_inputs(case, seed)
    rows = [x.table[b, :x.held[b]].tolist() for b in range(x.slots)]
    ctx, refs = x.ctx.tolist(), x.refs.tolist()
    copies, live = [], None
    if case["kind"] == "branch":
        for a, b in zip(x.src.tolist(), x.dst.tolist()):
            rows[b], ctx[b] = rows[a][:-(-ctx[a] // BLOCK)], ctx[a]
            for i in rows[b]:
                refs[i] += 1
        before = list(refs)
        free = iter([i for i, c in enumerate(before) if c == 0])
        for b, t in enumerate(x.tokens.tolist()):
            for at in range(ctx[b] // BLOCK, -(-t // BLOCK)):
                if at < len(rows[b]) and before[rows[b][at]] == 1:
                    continue
                new = next(free)
                refs[new] = 1
                if at < len(rows[b]):
                    refs[rows[b][at]] -= 1
                    if at * BLOCK < ctx[b]:
                        copies.append((rows[b][at], new))
                    rows[b][at] = new
                else:
                    rows[b].append(new)
    else:
        for b in x.gone.tolist():
            for i in rows[b]:
                refs[i] -= 1
            rows[b], ctx[b] = [], 0
        live = sum(c > 0 for c in refs)
        copies = list(zip([i for i, c in enumerate(refs) if c > 0 and i >= live], [i for i, c in enumerate(refs) if c == 0 and i < live]))
        move = dict(copies)
        for a, b in copies:
            refs[a], refs[b] = 0, refs[a]
        rows = [[move.get(i, i) for i in r] for r in rows]
    table = np.full((x.slots, x.width), -1, np.int32)
    for b, r in enumerate(rows):
        table[b, :len(r)] = r
    k, v = _pages(case, case["layers"], x.blocks, seed)
    for t in (k, v):
        if copies:
            t[:, [b for _, b in copies]] = t[:, [a for a, _ in copies]]
    got = {"table": _i32(table), "refs": _i32(refs), "held": _i32([len(r) for r in rows]), "ctx": _i32(ctx), "k": k.double(), "v": v.double()}
    if live is not None:
        got["live"] = _i32([live])
    return got


def exact(case, seed):
    return {"prompt": _exact_prompt, "prefix": _exact_prefix, "pages": _exact_pages}[case["op"]](case, seed)
