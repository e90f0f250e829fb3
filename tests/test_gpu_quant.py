"""GPU parity of the cache held in 4 bits (kvr_quant_append, kvr_quant_read) and
of the attention over it (kvr_quant_attn) against oracle/quant.py.

Appends are exact: what is read back equals the oracle's values, rounded to the
destination's type. Attention, bfloat16: an output is rounded by at most 2^-8
of itself; inside, probabilities, their products with a scale, and the partial
outputs that splits leave are float16 (half a step 2^-11 each), and s n may be
twice as large as a value, so 8 x 2^-11 of the largest |v| covers the rest with
float32's rounding errors. float32: logits of |q||k| D terms and exps of them,
3e-5 of the largest |v|.
"""
import math

import numpy as np
import pytest
import torch

from gpu_util import as_f64, say
from oracle import quant as oq

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def kvr():
    from paper_2608_15797_amd import kvr as k
    return k


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def normal(shape, seed, dtype=BF, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def garbage(cache, seed):
    """Every byte set: float16 NaNs among the scales and offsets of slots that nothing has written."""
    g = torch.Generator().manual_seed(seed)
    cache.data.copy_(torch.randint(0, 256, cache.data.shape, generator=g, dtype=torch.uint8))
    cache.data[..., -256:] = 0xff
    return cache


def read(cache, S, cap, lens, dtype=F32):
    k = kvr()
    _, L, Hkv = cache.data.shape[:3]
    dst = k.Cache(torch.full((S, L, Hkv, cap, cache.D), -7.0, dtype=dtype, device=DEV),
                  torch.full((S, L, Hkv, cap, cache.D), -7.0, dtype=dtype, device=DEV))
    k.quant_read(cache, dst, lens)
    torch.cuda.synchronize()
    return dst


CASES = [  # S, L, Hkv, cap, T, len, count
    (3, 2, 2, 100, 70, [0, 5, 31], [70, 0, 33]),
    (4, 1, 1, 64, 1, [0, 31, 32, 63], None),
    (2, 2, 1, 33, 40, [0, 20], [40, 40]),           # runs past the last slot
    (1, 1, 3, 1000, 513, [17], None),
    (2, 1, 1, 31, 8, [40, -3], [9, 5]),             # full already; lengths out of range
]


@pytest.mark.parametrize("D,group", [(128, 32), (128, 64), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_and_read_back(case, dtype, D, group):
    S, L, Hkv, cap, T, lens, counts = CASES[case]
    k = kvr()
    c = garbage(k.QuantCache.empty(S, L, Hkv, cap, D, group), case)
    old = [normal((S, L, Hkv, cap, D), 10 + i, F32).to(DEV) for i in range(2)]
    k.quant_append(c, ints([0] * S), k.Cache(*old))
    new = [normal((S, L, Hkv, T, D), 20 + i, dtype, 3.0) for i in range(2)]
    new[0][..., 5] *= 40.0
    k.quant_append(c, ints(lens), k.Cache(new[0].to(DEV), new[1].to(DEV)), count=None if counts is None else ints(counts))
    for to in (F32, BF):
        got = read(c, S, cap, ints([cap] * S), to)
        for g, o, x in zip((got.k, got.v), old, new):
            want = oq.stand_for(o.cpu().numpy(), group)
            xs = oq.stand_for(x.float().numpy(), group)
            for s in range(S):
                n, m = max(lens[s], 0), T if counts is None else min(max(counts[s], 0), T)
                m = max(0, min(m, cap - n))
                want[s, :, :, n:n + m] = xs[s, :, :, :m]
            assert torch.equal(g.cpu(), torch.from_numpy(want).to(F32).to(to))


def test_append_takes_rows_by_index_and_read_gives_them_by_index():
    k = kvr()
    src = [normal((3, 2, 2, 40, 128), 30 + i) for i in range(2)]
    c = garbage(k.QuantCache.empty(5, 2, 2, 50, 128), 1)
    before = c.data.clone()
    idx, cnt = [2, 0, 2, 3, -1], [40, 7, 33, 40, 40]
    k.quant_append(c, ints([0] * 5), k.Cache(src[0].to(DEV), src[1].to(DEV)), src_index=ints(idx), count=ints(cnt))
    torch.cuda.synchronize()
    assert torch.equal(c.data[3:], before[3:])      # indices outside the source are skipped
    dst = k.Cache.empty(4, 2, 2, 64, 128, F32, DEV, with_pos=False)
    dst.k.fill_(-7.0)
    dst.v.fill_(-7.0)
    k.quant_read(c, dst, ints([33, 7, 64, 40]), src_index=ints([2, 1, 9, 0]))
    torch.cuda.synchronize()
    for d, x in ((dst.k, src[0]), (dst.v, src[1])):
        v = torch.from_numpy(oq.stand_for(x.float().numpy(), 32)).float()
        d = d.cpu()
        assert torch.equal(d[0, :, :, :33], v[2, :, :, :33]) and torch.equal(d[1, :, :, :7], v[0, :, :, :7])
        assert torch.equal(d[3, :, :, :40], v[2, :, :, :40])
        assert (d[2] == -7).all() and (d[0, :, :, 33:] == -7).all() and (d[3, :, :, 40:] == -7).all()


def test_append_of_unusual_values():
    k = kvr()
    x = normal((1, 1, 1, 12, 64), 40, F32)
    x[..., 0, :32] = 3.25                                   # a constant group
    x[..., 1, 3] = float("nan")
    x[..., 2, 4], x[..., 2, 40] = float("inf"), float("-inf")
    x[..., 3, :] *= 1e-7                                    # scales below float16's smallest
    x[..., 4, :] *= 1e30                                    # clamped
    x[..., 5, :] = torch.arange(64) % 16                    # scale 1: ties below
    x[..., 6, :] = torch.arange(64) % 31 * 0.5
    x[..., 7, :] = 0.0
    x[..., 8, :] = -0.0
    x[..., 9, :] = 1000.0 + x[..., 9, :] * 1e-3
    x[..., 10, :] = float("nan")
    for dtype in (F32, BF):
        y = x.to(dtype)
        c = garbage(k.QuantCache.empty(1, 1, 1, 12, 64), 2)
        k.quant_append(c, ints([0]), k.Cache(y.to(DEV), y.flip(-1).contiguous().to(DEV)))
        got = read(c, 1, 12, ints([12]))
        for g, v in ((got.k, y), (got.v, y.flip(-1))):
            want = torch.from_numpy(oq.stand_for(v.float().numpy(), 32)).float()
            assert torch.isfinite(g).all() and torch.equal(g.cpu(), want)


@pytest.mark.parametrize("D,group", [(128, 32), (128, 64), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_appended_a_few_at_a_time_are_the_same_bytes(dtype, D, group):
    k = kvr()
    S, L, Hkv, T = 3, 2, 5, 57
    x = [normal((S, L, Hkv, T, D), 50 + i, dtype) for i in range(2)]
    for y in x:
        y[:, :, 0, 3, 7], y[:, :, 1, 20, 9], y[:, :, 1, 21, 10] = float("nan"), float("inf"), float("-inf")
        y[:, :, 2, 30] *= 1e30
        y[:, :, 3, 40] = -0.0
        y[:, :, 3, 41, ::2] = 0.0
        y[:, :, 3, 41, 1::2] = -0.0
        y[:, :, 4, 42] = float("nan")
    x = [y.to(DEV) for y in x]
    start = ints([0, 9, 40])
    whole = garbage(k.QuantCache.empty(S, L, Hkv, 90, D, group), 3)
    parts = garbage(k.QuantCache.empty(S, L, Hkv, 90, D, group), 3)
    assert torch.equal(whole.data, parts.data)
    k.quant_append(whole, start, k.Cache(*x))
    a = 0
    for n in (1, 2, 16, 3, 17, 8, 10):
        k.quant_append(parts, start + a, k.Cache(*(y[:, :, :, a:a + n].contiguous() for y in x)))
        a += n
    torch.cuda.synchronize()
    assert a == T and torch.equal(whole.data, parts.data)


def build(P, L, Hkv, D, group, lens, cap, seed, dtype=BF):
    """A context cache whose unwritten slots are garbage, and its values."""
    k = kvr()
    c = garbage(k.QuantCache.empty(P, L, Hkv, cap, D, group), seed)
    n = max(max(lens), 1)
    rows = [normal((P, L, Hkv, n, D), seed + i, dtype) for i in range(2)]
    k.quant_append(c, ints([0] * P), k.Cache(rows[0].to(DEV), rows[1].to(DEV)), count=ints(lens))
    return c, [oq.stand_for(r.float().numpy(), group) for r in rows]


def roomy(ctx, tiles):
    """The same context at the front of units of that many tiles."""
    S, L, Hkv, held, _ = ctx.data.shape
    big = kvr().QuantCache.empty(S, L, Hkv, 32 * tiles, ctx.D, ctx.group)
    big.data.fill_(0xff)
    big.data[:, :, :, :held] = ctx.data
    return big


def check(got, ref, vmax, dtype, what, more=0.0):
    err = np.abs(got - ref)
    tol = 2.0 ** -8 * np.abs(ref) + (8 * 2.0 ** -11 + more) * vmax if dtype == BF else 3e-5 * vmax + 0 * ref
    say(what, "largest error / tolerance %.3f" % (err / np.maximum(tol, 1e-30)).max(),
        "rms error / rms %.2e" % (np.sqrt((err ** 2).mean()) / max(np.sqrt((ref ** 2).mean()), 1e-30)))
    assert np.isfinite(got).all() and (err <= tol).all()


ATTN = [  # P, C, L, G, Hkv, D, group, nq, context lengths, own lengths (None: no own cache)
    (3, 1, 2, 6, 2, 128, 32, 1, [0, 1, 33], [1, 64, 17]),
    (2, 1, 1, 6, 2, 128, 64, 1, [4096, 1337], [1, 130]),
    (2, 3, 2, 7, 1, 128, 32, 1, [500, 97], [3, 1, 40, 33, 32, 31]),
    (1, 8, 1, 6, 2, 128, 64, 1, [2049], [1, 2, 3, 4, 5, 6, 7, 80]),
    (2, 1, 2, 7, 4, 128, 32, 5, [700, 64], [5, 37]),
    (2, 1, 1, 8, 8, 128, 64, 3, [32, 31], None),
    (5, 1, 1, 4, 2, 64, 32, 2, [0, 1, 2, 3, 300], None),
    (3, 1, 1, 16, 1, 64, 64, 4, [100, 0, 8], [4, 2, 0]),
    (1, 1, 1, 1, 1, 64, 32, 1, [1], None),
    (1, 1, 1, 16, 1, 128, 32, 64, [50], [20]),          # more rows than a block, queries into the context
    (1, 5, 1, 16, 1, 128, 32, 3, [333], [3, 9, 40, 41, 100]),
    (1, 1, 1, 8, 1, 128, 64, 1, [70001], [9]),
    (40, 2, 1, 2, 1, 64, 64, 1, list(range(0, 400, 10)), list(range(1, 81))),
]


def run_attn(case, dtype, new, seed=7, scale=None, tiles=0):
    P, C, L, G, Hkv, D, group, nq, lens, own = ATTN[case] if isinstance(case, int) else case
    k, S = kvr(), P * C
    ctx, (ck, cv) = build(P, L, Hkv, D, group, lens, max(lens) + 5, seed, dtype)
    if tiles:                    # the same contexts at the front of units of that many tiles
        ctx = roomy(ctx, tiles)
    q = normal((S, L, G * Hkv, nq, D), seed + 3, dtype)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = torch.full(q.shape, float("nan"), dtype=dtype, device=DEV)
    cache = kn = vn = lt = pos = None
    if own is not None:
        cap = max(own) + 3
        ok, ov = normal((S, L, Hkv, cap, D), seed + 4, dtype), normal((S, L, Hkv, cap, D), seed + 5, dtype)
        for s in range(S):       # slots past the last live one hold anything
            ok[s, :, :, own[s]:] = float("nan")
            ov[s, :, :, own[s]:] = float("inf")
        cache = k.Cache(ok.to(DEV), ov.to(DEV), torch.full((S, L, Hkv, cap), -1, dtype=torch.int32, device=DEV))
        lt = ints(own)
        if new:
            kn, vn = normal((S, L, Hkv, nq, D), seed + 6, dtype), normal((S, L, Hkv, nq, D), seed + 8, dtype)
            pos = torch.arange(S * nq, dtype=torch.int32).view(S, nq)
    nb = k.quant_attn_workspace_size(ctx, cache, G * Hkv, nq, dtype)
    ws = torch.full((max(nb, 16) // 4 + 4,), float("nan"), device=DEV)
    k.quant_attn(ctx, ints(lens), q.to(DEV), out, scale, own=cache, len_=lt,
                 k_new=None if kn is None else kn.to(DEV), v_new=None if vn is None else vn.to(DEV),
                 new_pos=None if pos is None else pos.to(DEV), workspace=ws)
    torch.cuda.synchronize()
    got = as_f64(out)
    ref = np.zeros(got.shape)
    vmax = np.zeros(got.shape[:3] + (1, 1))
    for s in range(S):
        n = lens[s // C]
        kk, vv = ck[s // C][:, :, :n], cv[s // C][:, :, :n]
        if own is not None:
            ko, vo = as_f64(ok)[s].copy(), as_f64(ov)[s].copy()
            if new:
                for t in range(nq):
                    j = own[s] - nq + t
                    if j >= 0:
                        ko[:, :, j], vo[:, :, j] = as_f64(kn)[s, :, :, t], as_f64(vn)[s, :, :, t]
            # The cache holds the new rows, and nothing else has changed.
            for a, b in ((cache.k, ko), (cache.v, vo)):
                assert np.array_equal(as_f64(a)[s], b, equal_nan=True)
            p = cache.pos[s].cpu().numpy()
            for j in range(cap):
                t = j - (own[s] - nq)
                assert (p[:, :, j] == (int(pos[s, t]) if new and 0 <= t < nq else -1)).all()
            kk, vv = np.concatenate([kk, ko[:, :, :own[s]]], 2), np.concatenate([vv, vo[:, :, :own[s]]], 2)
        for l in range(L):
            for h in range(Hkv):
                hs = slice(h * G, (h + 1) * G)
                ref[s, l, hs] = oq.attend(kk[l, h], vv[l, h], as_f64(q)[s, l, hs], scale)
                vmax[s, l, hs] = np.abs(vv[l, h]).max() if vv.shape[2] else 0.0
    check(got, ref, vmax, dtype, (case if isinstance(case, int) else "case", str(dtype), new))
    return got


@pytest.mark.parametrize("new", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(case, dtype, new):
    if new and ATTN[case][9] is None:
        pytest.skip("no own cache to append to")
    run_attn(case, dtype, new)


@pytest.mark.parametrize("D,group", [(128, 32), (128, 64), (64, 32), (64, 64)])
@pytest.mark.parametrize("G,nq", [(5, 1), (5, 4), (5, 8), (5, 12)])
def test_every_number_of_row_blocks(G, nq, D, group):
    """One to four blocks of 16 query rows in each layout, over tiles that are full, cut and crossed."""
    run_attn((2, 1, 2, G, 2, D, group, nq, [259, 31], [nq, nq + 30]), BF, True)
    run_attn((2, 1, 2, G, 2, D, group, nq, [259, 31], None), BF, False)


@pytest.mark.parametrize("D,group", [(128, 32), (128, 64), (64, 32), (64, 64)])
@pytest.mark.parametrize("G,nq", [(5, 1), (5, 4), (5, 8), (5, 12), (7, 14), (5, 30)])
def test_row_blocks_of_a_wave_over_caches_of_many_tiles(G, nq, D, group):
    """The same rows where room for 65536 tiles and more gives a wave two blocks, three and four."""
    blocks = (G * nq + 15) // 16
    for room in (90000, 180000, 260000):
        tiles = room // (4 * blocks) + 1
        run_attn((2, 1, 1, G, 2, D, group, nq, [259, 31], [nq, nq + 30]), BF, True, tiles=tiles)
        run_attn((1, 2, 1, G, 4, D, group, nq, [300], [nq + 1, nq + 33]), BF, False, tiles=tiles)
        run_attn((2, 1, 1, G, 2, D, group, nq, [259, 31], None), BF, False, tiles=tiles)


@pytest.mark.parametrize("D,group", [(128, 32), (64, 64)])
@pytest.mark.parametrize("nq", [1, 3])
@pytest.mark.parametrize("new", [False, True])
def test_more_units_than_the_chip_has_waves(new, nq, D, group):
    """1040 units (and 280 of a tile each) of every length, some shorter than the query tokens."""
    lens, own = [(41 * i) % 75 for i in range(130)], [(29 * i) % 71 for i in range(260)]
    run_attn((130, 2, 1, 3, 4, D, group, nq, lens, own), BF, new)
    run_attn((140, 1, 1, 7, 2, D, group, nq, [i % 28 for i in range(140)], own[:140]), BF, new)
    if not new:
        run_attn((140, 1, 2, 6, 4, D, group, nq, [i % 28 for i in range(140)], None), BF, False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_more_contexts_than_lanes(dtype):
    lens = [(37 * i * i) % 201 if i % 9 else 0 for i in range(150)]
    run_attn((150, 1, 2, 3, 1, 64, 32, 1, lens, [1 + i % 40 for i in range(150)]), dtype, True)
    run_attn((150, 2, 1, 2, 2, 64, 64, 2, lens, [2 + i % 5 for i in range(300)]), dtype, False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_of_sharp_and_of_flat_logits(dtype):
    # Logits of +-100 (one key decides) and of 0 (all count alike).
    run_attn((2, 2, 1, 6, 2, 128, 32, 2, [300, 64], [2, 40, 3, 9]), dtype, True, scale=1.0)
    run_attn((2, 2, 1, 6, 2, 128, 32, 2, [300, 64], [2, 40, 3, 9]), dtype, True, scale=0.0)


def test_lengths_past_the_caches_count_as_full():
    k = kvr()
    ctx, _ = build(2, 1, 2, 128, 32, [40, 40], 40, 50)
    own = k.Cache(normal((2, 1, 2, 9, 128), 51).to(DEV), normal((2, 1, 2, 9, 128), 52).to(DEV))
    q = normal((2, 1, 12, 1, 128), 53).to(DEV)
    res = []
    for cl, ol in (([40, 0], [9, 0]), ([99, -5], [12, -1])):
        out = torch.empty_like(q)
        ws = torch.empty(k.quant_attn_workspace_size(ctx, own, 12) + 16, dtype=torch.uint8, device=DEV)
        k.quant_attn(ctx, ints(cl), q, out, 0.1, own=own, len_=ints(ol), workspace=ws)
        torch.cuda.synchronize()
        res.append(out.cpu())
    assert torch.equal(res[0], res[1]) and (res[0][1] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_later_tokens_nan_does_not_reach_earlier_queries(dtype):
    """Four query tokens; the third's key and the last's value are NaN and infinite: the first two see neither."""
    k = kvr()
    P, L, Hkv, G, D, nq, u = 2, 1, 2, 4, 128, 4, 21
    ctx, (ck, cv) = build(P, L, Hkv, D, 32, [77, 0], 80, 60, dtype)
    ok, ov = normal((P, L, Hkv, u, D), 61, dtype), normal((P, L, Hkv, u, D), 62, dtype)
    kn, vn = normal((P, L, Hkv, nq, D), 63, dtype), normal((P, L, Hkv, nq, D), 64, dtype)
    kn[:, :, :, 2, 5] = float("nan")
    vn[:, :, :, 3, ::2] = float("inf")
    vn[:, :, :, 3, 1::2] = float("nan")
    q = normal((P, L, G * Hkv, nq, D), 65, dtype)
    out = torch.empty(q.shape, dtype=dtype, device=DEV)
    cache = k.Cache(ok.to(DEV), ov.to(DEV))
    ws = torch.empty(k.quant_attn_workspace_size(ctx, cache, G * Hkv, nq, dtype) + 16, dtype=torch.uint8, device=DEV)
    k.quant_attn(ctx, ints([77, 0]), q.to(DEV), out, 0.1, own=cache, len_=ints([u, u]), k_new=kn.to(DEV),
                 v_new=vn.to(DEV), workspace=ws)
    torch.cuda.synchronize()
    got = as_f64(out)
    assert not np.isfinite(got[..., 2:, :]).any()
    for p in range(P):
        n = [77, 0][p]
        for h in range(Hkv):
            kk = np.concatenate([ck[p][0, h][:n], as_f64(ok)[p, 0, h, :u - nq], as_f64(kn)[p, 0, h, :2]])
            vv = np.concatenate([cv[p][0, h][:n], as_f64(ov)[p, 0, h, :u - nq], as_f64(vn)[p, 0, h, :2]])
            hs = slice(h * G, (h + 1) * G)
            ref = oq.attend(kk, vv, as_f64(q)[p, 0, hs][:, :2], 0.1)
            check(got[p, 0, hs][:, :2], ref, np.abs(vv).max(), dtype, "masked NaN")


@pytest.mark.parametrize("std", [1e-4, 30.0, 3000.0])
def test_attention_of_small_and_large_values(std):
    """Values far from 1: errors stay relative to the largest value."""
    k = kvr()
    P, L, Hkv, G, D = 1, 1, 1, 6, 128
    rows = [normal((P, L, Hkv, 700, D), 70, F32), normal((P, L, Hkv, 700, D), 71, F32, std)]
    ctx = garbage(k.QuantCache.empty(P, L, Hkv, 700, D, 32), 3)
    k.quant_append(ctx, ints([0]), k.Cache(rows[0].to(DEV), rows[1].to(DEV)))
    q = normal((P, L, G, 1, D), 72)
    out = torch.empty(q.shape, dtype=BF, device=DEV)
    ws = torch.empty(k.quant_attn_workspace_size(ctx, None, G) + 16, dtype=torch.uint8, device=DEV)
    k.quant_attn(ctx, ints([700]), q.to(DEV), out, 0.09, workspace=ws)
    torch.cuda.synchronize()
    kk, vv = (oq.stand_for(r.numpy(), 32)[0, 0, 0] for r in rows)
    ref = oq.attend(kk, vv, as_f64(q)[0, 0], 0.09)
    check(as_f64(out)[0, 0], ref, np.abs(vv).max(), BF, ("std", std))


@pytest.mark.parametrize("std", [1e-6, 1e4])
def test_attention_of_small_and_large_queries(std):
    """Queries whose size the scale undoes, far outside float16's range."""
    k = kvr()
    ctx, (ck, cv) = build(1, 1, 1, 128, 64, [333], 333, 80)
    q = normal((1, 1, 6, 2, 128), 82, BF, std)
    q[..., 7] *= 100.0
    own = k.Cache(normal((1, 1, 1, 40, 128), 83).to(DEV), normal((1, 1, 1, 40, 128), 84).to(DEV))
    out = torch.empty(q.shape, dtype=BF, device=DEV)
    ws = torch.empty(k.quant_attn_workspace_size(ctx, own, 6, 2) + 16, dtype=torch.uint8, device=DEV)
    sc = 0.02 / std
    k.quant_attn(ctx, ints([333]), q.to(DEV), out, sc, own=own, len_=ints([40]), workspace=ws)
    torch.cuda.synchronize()
    kk = np.concatenate([ck[0][0, 0], as_f64(own.k)[0, 0, 0]])
    vv = np.concatenate([cv[0][0, 0], as_f64(own.v)[0, 0, 0]])
    check(as_f64(out)[0, 0], oq.attend(kk, vv, as_f64(q)[0, 0], sc), np.abs(vv).max(), BF, ("q std", std))


@pytest.mark.parametrize("std,qstd,scale", [(1.0, 1.0, 1.0), (1.0, 1.0, 0.0), (1e-4, 1.0, 0.09), (3000.0, 1.0, 0.09),
                                            (1.0, 1e-6, 2e4), (1.0, 1e4, 2e-6)])
@pytest.mark.parametrize("G,nq,tiles", [(12, 2, 40000), (16, 3, 50000), (16, 4, 60000)])
@pytest.mark.parametrize("D,group", [(128, 32), (64, 64)])
def test_unusual_sizes_with_two_and_three_row_blocks(D, group, G, nq, tiles, std, qstd, scale):
    """Sharp and flat logits, values and queries far from 1. Three blocks and more take the keys' values as float16: each
    off by 2^-12 of itself, a logit by that of sum |q k|, and a probability by as much again through the sum."""
    k = kvr()
    rows = [normal((1, 1, 1, 333, D), 140, F32), normal((1, 1, 1, 333, D), 141, F32, std)]
    ctx = k.QuantCache.empty(1, 1, 1, 333, D, group)
    k.quant_append(ctx, ints([0]), k.Cache(rows[0].to(DEV), rows[1].to(DEV)))
    ctx = roomy(ctx, tiles)
    q = normal((1, 1, G, nq, D), 142, BF, qstd)
    q[..., 7] *= 10.0 if qstd != 1.0 else 1.0
    out = torch.empty(q.shape, dtype=BF, device=DEV)
    ws = torch.empty(k.quant_attn_workspace_size(ctx, None, G, nq), dtype=torch.uint8, device=DEV)
    k.quant_attn(ctx, ints([333]), q.to(DEV), out, scale, workspace=ws)
    torch.cuda.synchronize()
    kk, vv = (oq.stand_for(r.numpy(), group)[0, 0, 0] for r in rows)
    q = as_f64(q)[0, 0]
    more = 2 * 2.0 ** -12 * scale * (np.abs(q) @ np.abs(kk).T).max() if nq >= 3 else 0.0
    check(as_f64(out)[0, 0], oq.attend(kk, vv, q, scale), np.abs(vv).max(), BF, (D, G * nq, std, qstd, scale), more)


def _step(dtype=BF):
    """A call with its buffers: contexts shared by two candidates, three new tokens each."""
    k = kvr()
    P, C, L, Hkv, G, D, nq = 3, 2, 2, 2, 6, 128, 3
    S = P * C
    ctx, _ = build(P, L, Hkv, D, 32, [900, 0, 77], 901, 90, dtype)
    own = k.Cache(normal((S, L, Hkv, 50, D), 91, dtype).to(DEV), normal((S, L, Hkv, 50, D), 92, dtype).to(DEV))
    a = dict(q=normal((S, L, G * Hkv, nq, D), 93, dtype).to(DEV), kn=normal((S, L, Hkv, nq, D), 94, dtype).to(DEV),
             vn=normal((S, L, Hkv, nq, D), 95, dtype).to(DEV), cl=ints([900, 0, 77]), ol=ints([3, 50, 9, 33, 4, 12]))
    nb = k.quant_attn_workspace_size(ctx, own, G * Hkv, nq, dtype)
    a.update(ws=torch.empty(nb + 16, dtype=torch.uint8, device=DEV),
             out=torch.empty((S, L, G * Hkv, nq, D), dtype=dtype, device=DEV))

    def call(stream=None):
        k.quant_attn(ctx, a["cl"], a["q"], a["out"], 0.1, own=own, len_=a["ol"], k_new=a["kn"], v_new=a["vn"],
                     workspace=a["ws"], stream=stream)
    return call, a, ctx, own


def test_attention_repeats_bit_for_bit_on_any_stream():
    call, a, _, _ = _step()
    call()
    torch.cuda.synchronize()
    ref = a["out"].clone()
    side = torch.cuda.Stream()
    for st in (None, side, side):
        a["out"].fill_(0)
        a["ws"].fill_(0xff)
        torch.cuda.synchronize()
        call(st)
        torch.cuda.synchronize()
        assert torch.equal(a["out"].view(torch.int16), ref.view(torch.int16))


def test_captured_step_follows_lengths_that_change_between_replays():
    """Append, attention and read in one graph; the lengths are device data, so replays follow them."""
    k = kvr()
    call, a, ctx, own = _step()
    count = ints([0, 5, 0])
    dst = k.Cache.empty(3, 2, 2, 901, 128, F32, DEV, with_pos=False)

    def step():
        k.quant_append(ctx, a["cl"], own, src_index=ints_idx, count=count)
        call()
        k.quant_read(ctx, dst, a["cl"])
    ints_idx = ints([0, 3, 5])
    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    for rep, (cl, ol) in enumerate([([900, 0, 77], [3, 50, 9, 33, 4, 12]), ([10, 5, 0], [50, 3, 3, 40, 7, 8]),
                                    ([901, 901, 901], [20, 20, 20, 20, 20, 20])]):
        got = []
        for how in (step, graph.replay):
            a["cl"].copy_(ints(cl))
            a["ol"].copy_(ints(ol))
            a["out"].fill_(0)
            dst.k.fill_(0)
            dst.v.fill_(0)
            torch.randn(1 << 20, device="cuda").sum()
            torch.cuda.synchronize()
            how()
            torch.cuda.synchronize()
            # Bit patterns: the last lengths take in slots that nothing has written.
            got.append([t.clone() for t in (a["out"].view(torch.int16), dst.k.view(torch.int32), dst.v.view(torch.int32))])
        for x, y in zip(*got):
            assert torch.equal(x, y), rep


def test_two_calls_at_once_with_their_own_workspaces():
    pairs = [_step(), _step()]
    for call, *_ in pairs:
        call()
    torch.cuda.synchronize()
    ref = [p[1]["out"].clone() for p in pairs]
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(3):
        for (call, *_), st in zip(pairs, streams):
            call(st)
    torch.cuda.synchronize()
    for (_, a, _, _), r in zip(pairs, ref):
        assert torch.equal(a["out"].view(torch.int16), r.view(torch.int16))


def test_a_cache_of_some_sequences_is_the_same_memory():
    k = kvr()
    ctx, (ck, _) = build(4, 2, 2, 64, 32, [33, 64, 1, 50], 64, 100)
    got = read(ctx.sequences(1, 3), 2, 64, ints([64, 1]))
    assert torch.equal(got.k[0].cpu(), torch.from_numpy(ck[1][:, :, :64]).float())
    assert torch.equal(got.k[1, :, :, :1].cpu(), torch.from_numpy(ck[2][:, :, :1]).float())


def test_context_past_4_gib():
    """Offsets past 32 bits: the last of 60 units of 80 MB holds the live rows."""
    k = kvr()
    P, cap = 60, 1 << 19
    c = k.QuantCache.empty(P, 1, 1, cap, 128, 32)
    assert c.data.numel() > (1 << 32)
    rows = [normal((1, 1, 1, 50, 128), 110 + i) for i in range(2)]
    src = k.Cache(rows[0].to(DEV), rows[1].to(DEV))
    lens = [0] * P
    lens[P - 1], lens[P // 2] = cap - 50, 7
    cnt = [0] * P
    cnt[P - 1] = cnt[P // 2] = 50
    k.quant_append(c, ints(lens), src, src_index=ints([0] * P), count=ints(cnt))
    small = k.QuantCache.empty(1, 1, 1, 64, 128, 32)
    k.quant_append(small, ints([0]), src)
    dst = k.Cache.empty(1, 1, 1, cap, 128, F32, DEV, with_pos=False)
    k.quant_read(c, dst, ints([cap]), src_index=ints([P - 1]))
    want = read(small, 1, 50, ints([50]))
    torch.cuda.synchronize()
    assert torch.equal(dst.k[0, 0, 0, cap - 50:], want.k[0, 0, 0]) and torch.equal(dst.v[0, 0, 0, cap - 50:], want.v[0, 0, 0])
    # Attention over the rows at the front of the last context.
    k.quant_append(c, ints([0] * P), src, src_index=ints([0] * P), count=ints([0] * (P - 1) + [50]))
    q = normal((P, 1, 6, 1, 128), 120).to(DEV)
    for dtype in (BF, F32):
        qd, out = q.to(dtype), torch.empty(q.shape, dtype=dtype, device=DEV)
        ws = torch.empty(k.quant_attn_workspace_size(c, None, 6, 1, dtype) + 16, dtype=torch.uint8, device=DEV)
        k.quant_attn(c, ints([0] * (P - 1) + [50]), qd, out, 0.09, workspace=ws)
        torch.cuda.synchronize()
        assert (out[:P - 1] == 0).all()
        kk, vv = as_f64(want.k)[0, 0, 0], as_f64(want.v)[0, 0, 0]
        check(as_f64(out)[P - 1, 0], oq.attend(kk, vv, as_f64(qd)[P - 1, 0], 0.09), np.abs(vv).max(), dtype, "4 GiB")


def test_own_cache_of_rows_past_4_gib():
    """2^24 + 100 own rows of 256 bytes; those that carry the weight are read where all that are left are 4 GiB."""
    k = kvr()
    n, lo, hi = (1 << 24) + 100, 70, 100
    own = k.Cache(torch.zeros((1, 1, 1, n, 128), dtype=BF, device=DEV), torch.zeros((1, 1, 1, n, 128), dtype=BF, device=DEV))
    v = normal((hi - lo, 128), 130)
    own.k[0, 0, 0, lo:hi] = 0.5                      # logits of 40 among zeros: 30 e^40 to 2^24
    own.v[0, 0, 0, lo:hi] = v.to(DEV)
    c = k.QuantCache.empty(1, 1, 1, 32, 128, 32)
    q = torch.ones((1, 1, 2, 1, 128), dtype=BF, device=DEV)
    out = torch.empty_like(q)
    ws = torch.empty(k.quant_attn_workspace_size(c, own, 2, 1, BF), dtype=torch.uint8, device=DEV)
    k.quant_attn(c, ints([0]), q, out, 40.0 / 64, own=own, len_=ints([n]), workspace=ws)
    torch.cuda.synchronize()
    want = as_f64(v).mean(0)
    check(as_f64(out)[0, 0], np.broadcast_to(want, (2, 1, 128)), np.abs(as_f64(v)).max(), BF, "long own")
