"""Attention over whole prompts (mn_prompt_attention) against the definition in 64 bits, every element within the bound that the
roundings of its inputs' type allow (attention_bounds.py)."""
import numpy as np
import pytest
import torch

from paper_2402_15678_amd import synth
from tests.attention_bounds import attend, check, factors, levels, ties

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "f32": torch.float32}


def _model(H, Hkv, hd, kind, max_pos=1 << 16):
    from paper_2402_15678_amd import harness
    d = synth.ModelDesc(synth.ARCH_LLAMA, synth.DT_BF16 if kind == "f16" else synth.DT_F32, 1, 128, H, Hkv, hd, 128, 8, max_pos)
    return d, harness.DeviceModel.random_on_device(d, 1)


def _rows(H, Hkv, hd, kind, lens, seed, scale=1.0, lead=0, tail=0, pad=0):
    """A QKV projection's rows; what lies in front of the first sequence and behind the last is not a number."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    M = lead + sum(lens)
    x = torch.randn((M + tail, (H + 2 * Hkv) * hd + pad), generator=g, device="cuda")
    x[:, :H * hd] *= scale
    x[:lead] = float("nan")
    x[M:] = float("nan")
    x[:, (H + 2 * Hkv) * hd:] = float("nan")
    x = x.to(DT[kind])
    q = x[:, :H * hd].view(-1, H, hd) if not pad else x[:, :H * hd].unflatten(1, (H, hd))
    k = x[:, H * hd:(H + Hkv) * hd].unflatten(1, (Hkv, hd))
    v = x[:, (H + Hkv) * hd:(H + 2 * Hkv) * hd].unflatten(1, (Hkv, hd))
    row0 = (lead + np.concatenate(([0], np.cumsum(lens)))).astype(np.int32)
    return q, k, v, row0


def _call(model, q, k, v, row0, out, kv=None, h_row0=None):
    from paper_2402_15678_amd import harness
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    harness.prompt_attention(model, q, k, v, torch.from_numpy(row0).cuda(), harness.PromptRows((row0 if h_row0 is None else h_row0).tolist()),
                             out, kv, 0, status)
    torch.cuda.synchronize()
    return status.item()


def _compare(q, k, v, row0, out, kind):
    for a, b in zip(row0[:-1].tolist(), row0[1:].tolist()):
        if a < b:
            want, bound = attend(q[a:b], k[a:b], v[a:b], torch.arange(b - a, device="cuda"), kind == "f16")
            check(out[a:b], want, bound)


GEOMETRIES = [(64, 8, 128, "f16"), (4, 4, 128, "f16"), (12, 12, 64, "f16"), (6, 2, 64, "f16"), (5, 1, 128, "f16"), (128, 2, 64, "f16"),
              (4, 4, 64, "f32"), (8, 2, 128, "f32"), (6, 2, 32, "f32"), (8, 8, 8, "f32"), (4, 1, 16, "f32"), (2, 2, 256, "f32"),
              (8, 8, 32, "f16"), (8, 2, 256, "f16"), (16, 4, 8, "f16"), (8, 8, 16, "f16")]


@pytest.mark.parametrize("H,Hkv,hd,kind", GEOMETRIES)
@pytest.mark.parametrize("lens", [[1], [2, 0, 1, 33], [15, 16, 17, 31, 32, 65], [130, 0, 257]], ids=str)
def test_prompt_matches_the_definition(H, Hkv, hd, kind, lens):
    d, model = _model(H, Hkv, hd, kind)
    q, k, v, row0 = _rows(H, Hkv, hd, kind, lens, sum(lens) + H + hd)
    out = torch.full((len(q), H * hd), -7.0, dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    _compare(q, k, v, row0, out, kind)


@pytest.mark.parametrize("H,Hkv,hd,kind,lens", [
    (64, 8, 128, "f16", [700, 1, 1153, 64]), (8, 8, 128, "f16", [2100, 300, 3]), (12, 12, 64, "f16", [1500, 77, 512, 513]),
    (64, 8, 128, "f16", [5]), (40, 40, 128, "f16", [300, 900, 60, 777]), (8, 1, 64, "f16", [4099]), (4, 4, 64, "f32", [1000, 31]), (24, 2, 64, "f16", [1, 4000, 2])])
def test_long_and_ragged_prompts(H, Hkv, hd, kind, lens):
    d, model = _model(H, Hkv, hd, kind)
    q, k, v, row0 = _rows(H, Hkv, hd, kind, lens, 5)
    out = torch.full((len(q), H * hd), -7.0, dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    _compare(q, k, v, row0, out, kind)


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("count", [64, 65, 300, 4096])
def test_many_sequences(kind, hd, count):
    g = np.random.default_rng(count)
    lens = [int(x) for x in (g.integers(0, 9, count) if count > 300 else g.integers(0, 120, count))]
    d, model = _model(4, 2, hd, kind)
    q, k, v, row0 = _rows(4, 2, hd, kind, lens, 6)
    out = torch.full((len(q), 4 * hd), -7.0, dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    # (a sample of the sequences: the definition goes one by one)
    for b in sorted(set(g.integers(0, count, 60).tolist())):
        a, z = int(row0[b]), int(row0[b + 1])
        if a < z:
            check(out[a:z], *attend(q[a:z], k[a:z], v[a:z], torch.arange(z - a, device="cuda"), kind == "f16"))
    assert not (out == -7.0).all(dim=1).any()


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f16", 64), ("f32", 32), ("f16", 32)])
def test_rows_outside_the_sequences_are_neither_read_nor_written(kind, hd):
    lens, lead, tail = [70, 5, 129], 3, 9
    d, model = _model(8, 4, hd, kind)
    q, k, v, row0 = _rows(8, 4, hd, kind, lens, 7, lead=lead, tail=tail, pad=16)
    out = torch.full((len(q), 8 * hd), -7.0, dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    _compare(q, k, v, row0, out, kind)
    assert (out[:lead] == -7.0).all() and (out[lead + sum(lens):] == -7.0).all()


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("shape", ["peaked", "rising", "falling", "flat", "late"])
def test_scores_far_apart(kind, hd, shape):
    """The running reference: scores of +-200 and more, ascending and descending along the keys, all equal, one large one late."""
    n = 300
    d, model = _model(4, 2, hd, kind)
    q, k, v, row0 = _rows(4, 2, hd, kind, [n], 8)
    q, k = q.clone(), k.clone()
    if shape == "peaked":
        q *= 20
    elif shape in ("rising", "falling"):
        q[:] = 1.0
        ramp = torch.arange(n, device="cuda") / n * 40 - 20
        k[:] = (ramp if shape == "rising" else ramp.flip(0)).view(-1, 1, 1).to(k.dtype)
    elif shape == "flat":
        k[:] = 0.0
    else:
        q[:] = 4.0
        k *= 0.1
        k[n - 70] = 8.0
    out = torch.zeros((n, 4 * hd), dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    _compare(q, k, v, row0, out, kind)


def test_values_of_the_whole_fp16_range():
    for hd in (64, 128, 32):
        d, model = _model(4, 4, hd, "f16")
        q, k, v, row0 = _rows(4, 4, hd, "f16", [100], 9)
        v = torch.where(v > 0, 65504.0, -65504.0).to(torch.float16)
        v[:, 1] = 6e-8
        out = torch.zeros((100, 4 * hd), dtype=torch.float16, device="cuda")
        assert _call(model, q, k, v, row0, out) == 0
        _compare(q, k, v, row0, out, "f16")


@pytest.mark.parametrize("H,Hkv,hd,kind,bs", [(64, 8, 128, "f16", 16), (6, 2, 64, "f16", 16), (4, 4, 64, "f32", 16), (4, 2, 128, "f16", 8),
                                              (6, 2, 32, "f32", 5), (8, 8, 8, "f32", 1), (5, 1, 128, "f16", 16)])
def test_prompts_enter_the_cache(H, Hkv, hd, kind, bs):
    from paper_2402_15678_amd import harness
    lens = [37, 1, 0, 64, 130]
    d, model = _model(H, Hkv, hd, kind)
    q, k, v, row0 = _rows(H, Hkv, hd, kind, lens, 10)
    need = [-(-n // bs) for n in lens]
    g = np.random.default_rng(3)
    ids = g.permutation(sum(need) + 3).astype(np.int32)
    table = np.full((len(lens), max(need) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    blocks = len(ids)
    kp = torch.full((blocks, Hkv, hd // 8, bs, 8), -3.0, dtype=DT[kind], device="cuda")
    vp = torch.full((blocks, Hkv, hd, bs), -3.0, dtype=DT[kind], device="cuda")
    wk, wv = kp.clone(), vp.clone()
    for b, n in enumerate(lens):
        for i in range(n):
            r, blk, off = int(row0[b]) + i, int(table[b, i // bs]), i % bs
            wk[blk, :, :, off] = k[r].view(Hkv, -1, 8)
            wv[blk, :, :, off] = v[r]
    kv = harness.DeviceKV(d, bs, blocks, table, [9] * len(lens), [kp], [vp])
    out = torch.zeros((len(q), H * hd), dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out, kv) == 0
    _compare(q, k, v, row0, out, kind)
    assert torch.equal(kp, wk) and torch.equal(vp, wv)
    assert kv.ctx_lens.tolist() == [9] * len(lens)
    # a block id out of range: its tokens stay out of the cache, everything else is as before
    from paper_2402_15678_amd import binding
    hit = int(table[4, 2 if bs > 1 else 100])
    table[4, 2 if bs > 1 else 100] = blocks + 5
    kp.fill_(-3.0)
    vp.fill_(-3.0)
    wk[hit], wv[hit] = -3.0, -3.0
    kv = harness.DeviceKV(d, bs, blocks, table, [9] * len(lens), [kp], [vp])
    again = torch.zeros_like(out)
    assert _call(model, q, k, v, row0, again, kv) == binding.MN_DEV_BLOCK_TABLE
    assert torch.equal(again, out) and torch.equal(kp, wk) and torch.equal(vp, wv)


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f32", 32)])
def test_lengths_that_do_not_fit_the_launch_leave_the_call_undone(kind, hd):
    from paper_2402_15678_amd import binding
    lens = [70, 40, 300]
    d, model = _model(4, 4, hd, kind)
    q, k, v, row0 = _rows(4, 4, hd, kind, lens, 11)
    for wrong in ([0, 70, 110, 411], [0, 70, 60, 410], [-1, 70, 110, 410], [0, 10, 20, 30], [0, 0, 0, 410], [0, 70, 110, 1 << 30]):
        out = torch.full((len(q), 4 * hd), -7.0, dtype=DT[kind], device="cuda")
        assert _call(model, q, k, v, np.array(wrong, np.int32), out, h_row0=row0) == binding.MN_DEV_SPEC_LEN
        assert (out == -7.0).all()


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f16", 64), ("f32", 32), ("f16", 32)])
@pytest.mark.parametrize("fill", [0, 70])
def test_a_sequence_longer_than_the_hosts_longest_leaves_the_call_undone(kind, hd, fill):
    """Rows that move between sequences within one number of tiles: the table's rows have no entry for the tokens beyond the host's
    longest sequence, so neither outputs nor pages may change.  (fill: more than 64 sequences, whose numbers are kept elsewhere.)"""
    from paper_2402_15678_amd import binding, harness
    bs, tile = (16, 64) if kind == "f16" and hd >= 64 else (4, 16)
    host = np.array([0, tile // 4, tile // 2] + [tile // 2] * fill, np.int32)
    moved = host.copy()
    moved[1] = tile // 2 - 1
    d, model = _model(4, 4, hd, kind)
    q, k, v, row0 = _rows(4, 4, hd, kind, np.diff(host).tolist(), 13)
    n, width = len(host) - 1, -(-(tile // 4) // bs)
    table = np.arange(n * width, dtype=np.int32).reshape(n, width)
    kp = torch.full((n * width, 4, hd // 8, bs, 8), -3.0, dtype=DT[kind], device="cuda")
    vp = torch.full((n * width, 4, hd, bs), -3.0, dtype=DT[kind], device="cuda")
    for cache in (None, harness.DeviceKV(d, bs, n * width, table, [0] * n, [kp], [vp])):
        out = torch.full((len(q), 4 * hd), -7.0, dtype=DT[kind], device="cuda")
        assert _call(model, q, k, v, moved, out, cache, h_row0=host) == binding.MN_DEV_SPEC_LEN
        assert (out == -7.0).all() and (kp == -3.0).all() and (vp == -3.0).all()
    assert _call(model, q, k, v, host, out, cache) == 0
    _compare(q, k, v, row0, out, kind)


def test_same_numbers_on_another_stream_and_from_a_graph():
    from paper_2402_15678_amd import harness
    d, model = _model(64, 8, 128, "f16")
    q, k, v, row0 = _rows(64, 8, 128, "f16", [300, 41, 800], 12)
    rows, plan = torch.from_numpy(row0).cuda(), harness.PromptRows(row0.tolist())
    want = torch.zeros((len(q), 64 * 128), dtype=torch.float16, device="cuda")
    harness.prompt_attention(model, q, k, v, rows, plan, want)
    out = torch.zeros_like(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        harness.prompt_attention(model, q, k, v, rows, plan, out)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        harness.prompt_attention(model, q, k, v, rows, plan, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        harness.prompt_attention(model, q, k, v, rows, plan, want)


def _same(got, want):
    """Bit for bit, NaN where there is NaN."""
    off = ~((got == want) | (got.isnan() & want.isnan()))
    assert not off.any().item(), f"{int(off.sum())} elements, the first (row, head, element) {off.nonzero()[0].tolist()}: {got[off][0].item()}, not {want[off][0].item()}"


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (4, 4, 128, "f16"), (12, 12, 64, "f16"), (6, 2, 64, "f16"), (4, 4, 64, "f32"), (8, 2, 128, "f32"),
                                           (8, 8, 8, "f32"), (2, 2, 256, "f32"), (8, 2, 256, "f16"), (8, 8, 32, "f16")])
@pytest.mark.parametrize("at", [0, 5, 40, 299])
def test_what_is_not_finite_reaches_the_rows_that_see_it(H, Hkv, hd, kind, at):
    """Infinities and NaN in a token's values: rows before it, other elements and other KV heads keep their bits, the rows from it on
    get what the sum is.  In its key: the rows from it on are not numbers.  In a query: its own row and head."""
    d, model = _model(H, Hkv, hd, kind)
    q, k, v, row0 = _rows(H, Hkv, hd, kind, [300, 7], 17)
    plain = torch.full((len(q), H * hd), -7.0, dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, plain) == 0
    plain = plain.view(-1, H, hd)
    G, h = H // Hkv, Hkv - 1
    odd = {1: float("inf"), 3: float("-inf"), 6: float("nan"), hd - 1: float("inf")}
    v2 = v.clone()
    for e, x in odd.items():
        v2[at, h, e] = x
    out = torch.empty_like(plain).view(-1, H * hd)
    assert _call(model, q, k, v2, row0, out) == 0
    want = plain.clone()
    for e, x in odd.items():
        want[at:300, h * G:, e] = x
    _same(out.view_as(want), want)

    k2 = k.clone()
    k2[at, h, 2] = float("nan")
    assert _call(model, q, k2, v, row0, out) == 0
    want = plain.clone()
    want[at:300, h * G:] = float("nan")
    _same(out.view_as(want), want)

    q2 = q.clone()
    q2[at, H - 1, 0] = float("nan")
    assert _call(model, q2, k, v, row0, out) == 0
    want = plain.clone()
    want[at, H - 1] = float("nan")
    _same(out.view_as(want), want)


@pytest.mark.parametrize("kind,hd,M,row", [("f16", 64, 140000, 16384), ("f16", 128, 80000, 32768), ("f32", 64, 40000, 32768)])
def test_rows_beyond_four_gigabytes(kind, hd, M, row):
    """Offsets of rows pass 32 bits: a short sequence, and a long one behind it, checked at rows all over it."""
    d, model = _model(2, 1, hd, kind)
    q, k, v, row0 = _rows(2, 1, hd, kind, [5, M - 5], 8, pad=row - 4 * hd)
    assert q.stride(0) == row and (M - 1) * row * q.element_size() > 1 << 32
    out = torch.full((M, 2 * hd), -7.0, dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    kk, vv = k[5:].contiguous(), v[5:].contiguous()
    for a in (0, 1, 31, 32, 127, 128, 1000, M // 2, M - 5 - 33, M - 6):
        rows = torch.arange(a, min(a + 2, M - 5), device="cuda")
        n = int(rows[-1]) + 1
        want, bound = attend(q[5:][rows], kk[:n], vv[:n], rows, kind == "f16")
        check(out[5:][rows], want, bound)


@pytest.mark.parametrize("kind,hd", [("f16", 128), ("f16", 64), ("f32", 64), ("f16", 256)])
@pytest.mark.parametrize("shape", ["rising", "falling", "any"])
@pytest.mark.parametrize("far", [True, False], ids=["far", "mixed"])
def test_prompt_scores_at_the_end_of_the_range(kind, hd, shape, far):
    n = 300
    d, model = _model(4, 2, hd, kind)
    q, k, v, row0 = _rows(4, 2, hd, kind, [n], 19)
    f = torch.full((n,), 65504.0 if kind == "f16" else 2.0 ** 53, device="cuda") if far else factors(n, kind, 3)
    q, k = q.clone(), k.clone()
    q[:] = f.view(-1, 1, 1).to(q.dtype)
    k[:] = (levels(n, shape, 4) * (8188.0 if kind == "f16" else 2.0 ** 50)).view(-1, 1, 1).to(k.dtype)
    out = torch.zeros((n, 4 * hd), dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    want, bound = ties(q, k, v, torch.arange(n, device="cuda"))
    check(out, want, bound + (2.0 ** -11 if kind == "f16" else 2.0 ** -24) * want.abs() + (2.0 ** -25 if kind == "f16" else 0))


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (12, 12, 64, "f16"), (4, 4, 64, "f32"), (8, 2, 256, "f16")])
def test_prompt_row_whose_scores_are_all_minus_infinity(H, Hkv, hd, kind):
    d, model = _model(H, Hkv, hd, kind)
    q, k, v, row0 = _rows(H, Hkv, hd, kind, [200, 7], 23)
    k = k.clone()
    k[:, :, 0] = -k[:, :, 0].abs() - 1
    plain = torch.empty((len(q), H * hd), dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, plain) == 0
    for at in (0, 63, 150):
        q2 = q.clone()
        q2[at, H - 1, 0] = float("inf")
        out = torch.empty_like(plain)
        assert _call(model, q2, k, v, row0, out) == 0
        want = plain.clone().view(-1, H, hd)
        want[at, H - 1] = float("nan")
        _same(out.view_as(want), want)


@pytest.mark.parametrize("H,Hkv,hd,kind", [(64, 8, 128, "f16"), (12, 12, 64, "f16"), (8, 8, 8, "f32"), (16, 4, 8, "f16"), (4, 1, 16, "f32"), (8, 2, 128, "f32"),
                                           (8, 2, 256, "f16")])
@pytest.mark.parametrize("at", [1, 40, 255])
def test_prompt_key_at_minus_infinity_has_no_weight(H, Hkv, hd, kind, at):
    """An infinity in one element of a key: a score of minus infinity, and the result without that key, where the query's element has the other
    sign; no number where it has the same."""
    n, e = 300, hd - 3
    d, model = _model(H, Hkv, hd, kind)
    q, k, v, row0 = _rows(H, Hkv, hd, kind, [n], 25)
    k = k.clone()
    k[at, :, e] = float("inf")
    out = torch.empty((n, H * hd), dtype=DT[kind], device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    rest = torch.arange(n, device="cuda") != at
    limit = torch.arange(n, device="cuda")
    want, bound = attend(q, k[rest], v[rest], limit - (limit >= at).long(), kind == "f16")
    up = ((limit >= at)[:, None] & (q[:, :, e] > 0))[:, :, None].expand(n, H, hd).reshape(n, -1)
    assert out[up].isnan().all() and up.any()
    check(torch.where(up, want.to(out.dtype), out), want, bound + 2.0 ** -11 * want.abs() + 2.0 ** -25)


@pytest.mark.parametrize("H,Hkv,hd,lens", [
    (4, 4, 128, [300, 65, 64, 63, 1, 0, 128]), (12, 12, 64, [300, 65, 64, 63, 1, 0, 128]),                       # tiles of 64 rows
    (40, 40, 128, [700, 1, 128, 0, 129, 127, 255, 400]), (64, 64, 64, [500, 33, 0, 128, 129, 1, 640]),           # tiles of 128 rows
    (64, 32, 128, [500, 65, 64, 1, 0, 463]), (48, 16, 128, [900, 43, 42, 1, 513]), (64, 32, 64, [801, 64, 65, 0, 400])], ids=str)
def test_every_row_of_a_tile_enters_the_cache(H, Hkv, hd, lens):
    """Heads of their own and small groups, the shapes with the most tokens per tile, at both tile heights, bit for bit."""
    from paper_2402_15678_amd import harness
    bs = 16
    d, model = _model(H, Hkv, hd, "f16")
    q, k, v, row0 = _rows(H, Hkv, hd, "f16", lens, 27)
    need = [-(-n // bs) for n in lens]
    ids = np.random.default_rng(4).permutation(sum(need) + 5).astype(np.int32)
    table = np.full((len(lens), max(need)), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = ids[sum(need[:b]):sum(need[:b + 1])]
    kp = torch.full((len(ids), Hkv, hd // 8, bs, 8), -3.0, dtype=torch.float16, device="cuda")
    vp = torch.full((len(ids), Hkv, hd, bs), -3.0, dtype=torch.float16, device="cuda")
    wk, wv = kp.clone(), vp.clone()
    for b, n in enumerate(lens):
        i = np.arange(n)
        blk, off = torch.from_numpy(table[b, i // bs].astype(np.int64)).cuda(), torch.from_numpy(i % bs).cuda()
        wk[blk, :, :, off] = k[row0[b]:row0[b + 1]].unflatten(2, (-1, 8))
        wv[blk, :, :, off] = v[row0[b]:row0[b + 1]]
    kv = harness.DeviceKV(d, bs, len(ids), table, [0] * len(lens), [kp], [vp])
    out = torch.full((len(q), H * hd), -7.0, dtype=torch.float16, device="cuda")
    assert _call(model, q, k, v, row0, out, kv) == 0
    assert torch.equal(kp, wk) and torch.equal(vp, wv)
    without = torch.empty_like(out)
    assert _call(model, q, k, v, row0, without) == 0
    assert torch.equal(out, without)
    _compare(q, k, v, row0, out, "f16")


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("scale", [60.0, 900.0, 14000.0])
def test_scores_of_any_size_give_a_mean_of_the_values_seen(hd, scale):
    """Random rows of up to the fp16 range: no score is known better than to its fp32 sum's rounding, but every output lies between the least
    and the largest value that its row sees (its own rounding aside)."""
    n = 300
    d, model = _model(4, 2, hd, "f16")
    q, k, v, row0 = _rows(4, 2, hd, "f16", [n], 28)
    q, k = (q.float() * scale).clamp(-65504, 65504).half(), (k.float() * scale).clamp(-65504, 65504).half()
    out = torch.zeros((n, 4 * hd), dtype=torch.float16, device="cuda")
    assert _call(model, q, k, v, row0, out) == 0
    assert torch.isfinite(out).all()
    seen = v.float().repeat_interleave(2, dim=1).reshape(n, -1)
    least, most = seen.cummin(dim=0).values, seen.cummax(dim=0).values
    # the weights of a row add up to 1 but for (n + 64) 2^-23, and the result is rounded by 2^-11
    slack = ((n + 64) * 2.0 ** -23 + 2.0 ** -11) * torch.maximum(least.abs(), most.abs()) + 2.0 ** -25
    assert (out.float() >= least - slack).all() and (out.float() <= most + slack).all()
