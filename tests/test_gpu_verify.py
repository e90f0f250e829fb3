"""GPU parity of kvr_verify_draft against oracle/quant.py, through the C ABI.

Decisions are taken in float64 on both sides, so counts, tokens and lengths are
equal; inputs are drawn so that no decision lies within 1e-9 of its border (the
margin the oracle reports is asserted).
"""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import quant as oq

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def kvr():
    from paper_2608_15797_amd import kvr as k
    return k


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def inputs(S, T, V, Vd, dtype, seed, kind="boosted", ld=None, ldd=None):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((S, T + 1, V), generator=g)
    if kind == "boosted":
        x *= 3.0
        idx = torch.randint(0, min(V, Vd or V), (S, T + 1, 6), generator=g)
        x.scatter_add_(2, idx, 8.0 + torch.randn(idx.shape, generator=g))
    elif kind == "ties":
        x = torch.randint(-3, 3, x.shape, generator=g).float()
    elif kind == "masked":
        x[torch.rand(x.shape, generator=g) < 0.99] = float("-inf")
        x[..., V // 2] = 0.0
    d = None
    if Vd:
        d = x[:, :T, :Vd] + torch.randn((S, T, Vd), generator=g)
        if kind == "ties":
            d = d.round()
    like = (d if d is not None else x[:, :T]).reshape(S * T, -1)
    w, ids = torch.topk(like, min(8, like.shape[1]), dim=1)
    pick = torch.multinomial(torch.softmax(w, 1), 1, generator=g)
    tok = ids.gather(1, pick).view(S, T).int()

    def pad(a, n):
        out = torch.full((a.shape[0] * a.shape[1], n), 77.0)   # what lies behind a row is larger than all of it
        out[:, :a.shape[2]] = a.reshape(-1, a.shape[2])
        return out.to(dtype)
    return (pad(x, ld or V), None if d is None else pad(d, ldd or Vd), tok, torch.rand((S, T), generator=g),
            torch.rand((S,), generator=g))


def run(x, d, tok, ua, ud, V, Vd, smp, dsmp=None, nd=None, lens=None, stream=None, seed=0):
    k = kvr()
    S, T = tok.shape
    top = max(smp[1], dsmp[1] if dsmp else 0)
    ws = torch.full((k.verify_draft_workspace_size(S, T, V, Vd, top) + 16,), 0xff, dtype=torch.uint8, device=DEV)
    acc, out = ints([-9] * S), torch.full((S, T + 1), -9, dtype=torch.int32, device=DEV)
    lt = None if lens is None else ints(lens)
    k.verify_draft(x.to(DEV), tok.to(DEV), k.Sampler(*smp), ua.to(DEV), ud.to(DEV), acc, out,
                   draft_logits=None if d is None else d.to(DEV), V=V, Vd=Vd if d is not None else None,
                   n_draft=None if nd is None else ints(nd), draft_sampler=k.Sampler(*dsmp) if dsmp else None,
                   len_=lt, len_out=lt, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    return acc.cpu().tolist(), out.cpu().tolist(), None if lt is None else lt.cpu().tolist()


def check(x, d, tok, ua, ud, V, Vd, smp, dsmp=None, nd=None, lens=None):
    S, T = tok.shape
    acc, out, after = run(x, d, tok, ua, ud, V, Vd, smp, dsmp, nd, lens)
    xs = x.float().numpy().reshape(S, T + 1, -1)[..., :V]
    ds = None if d is None else d.float().numpy().reshape(S, T, -1)[..., :Vd]
    least = np.inf
    for s in range(S):
        n = T if nd is None else min(max(nd[s], 0), T)
        res, margin = oq.verify(xs[s], None if ds is None else ds[s], tok[s].tolist(), n, ua[s].double().numpy(),
                                float(ud[s]), smp, dsmp)
        least = min(least, margin)
        assert margin > 1e-9, (s, margin)
        assert out[s] == res + [-1] * (T + 1 - len(res)), (s, out[s], res)
        assert acc[s] == len(res) - 1
        if lens is not None:
            assert after[s] == lens[s] - (n - acc[s])
    say("S", S, "T", T, "V", V, Vd, "accepted", sum(acc), "of", S * T, "least margin %.1e" % least)
    return acc


SMP = (0.8, 20, 0.95)


@pytest.mark.parametrize("S,T,V,Vd,dtype,kind", [
    (1, 1, 1, 0, BF, "flat"), (1, 4, 152064, 151936, BF, "boosted"), (7, 5, 32003, 32003, F32, "boosted"),
    (16, 3, 4099, 4000, BF, "ties"), (5, 2, 4099, 4099, F32, "ties"), (3, 32, 1000, 1000, BF, "boosted"),
    (9, 4, 50, 33, F32, "flat"), (6, 3, 2000, 2000, BF, "masked"), (300, 1, 700, 0, BF, "boosted"),
    (40, 5, 20000, 19000, BF, "flat")])
def test_tokens_counts_and_lengths(S, T, V, Vd, dtype, kind):
    x, d, tok, ua, ud = inputs(S, T, V, Vd, dtype, S * 100 + T, kind)
    check(x, d, tok, ua, ud, V, Vd, SMP)
    nd = [(3 * s) % (T + 3) - 1 for s in range(S)]      # from -1 to T + 1
    check(x, d, tok, ua, ud, V, Vd, SMP, nd=nd, lens=[100 + s for s in range(S)])


@pytest.mark.parametrize("top,dtop", [(1, 2), (2, 1), (3, 9), (9, 17), (17, 33), (33, 5), (64, 20), (20, 64)])
@pytest.mark.parametrize("V,dtype", [(200003, BF), (400000, F32), (700001, BF)])
def test_lists_of_many_splits(V, dtype, top, dtop):
    """Rows long enough for many splits, whose lists fill two merges' registers and more, of every list length."""
    x, d, tok, ua, ud = inputs(2, 2, V, V - 17, dtype, top * 100 + dtop, "boosted")
    check(x, d, tok, ua, ud, V, V - 17, (0.9, top, 1.0), (1.1, dtop, 1.0))
    x, _, tok, ua, ud = inputs(1, 2, V, 0, dtype, top * 100 + dtop + 1, "ties")
    check(x, None, tok, ua, ud, V, 0, (0.9, top, 1.0))


@pytest.mark.parametrize("smp,dsmp", [((1.0, 1, 1.0), None), ((0.3, 64, 1.0), (2.0, 3, 0.5)),
                                      ((1.7, 5, 0.1), (0.8, 64, 0.999))])
def test_samplers_of_their_own(smp, dsmp):
    x, d, tok, ua, ud = inputs(12, 4, 30001, 29000, BF, 5)
    check(x, d, tok, ua, ud, 30001, 29000, smp, dsmp)
    check(x, None, tok, ua, ud, 30001, 0, smp)


@pytest.mark.parametrize("ld,ldd", [(5003, 4801), (5008, 4808), (5001, 4900)])
def test_row_strides_and_unaligned_rows(ld, ldd):
    for dtype in (BF, F32):
        x, d, tok, ua, ud = inputs(4, 3, 5000, 4800, dtype, 6, ld=ld, ldd=ldd)
        check(x, d, tok, ua, ud, 5000, 4800, SMP)


def test_the_same_distributions_accept_everything_and_odd_tokens_never_stand():
    x, _, tok, ua, ud = inputs(8, 3, 9000, 0, BF, 8)
    d = x.view(8, 4, -1)[:, :3].reshape(24, -1).contiguous()
    # Tokens of the target's own nucleus: P = Q, u < 1, so all stand.
    for s in range(8):
        for t in range(3):
            ids = oq.distribution(d[3 * s + t].float().numpy(), *SMP)[0]
            tok[s, t] = int(ids[t % len(ids)])
    assert check(x, d, tok, ua, ud, 9000, 9000, SMP) == [3] * 8
    bad = tok.clone()
    bad[0, 0], bad[1, 1], bad[2, 2], bad[3, 0] = -1, 9000, 1 << 30, int(x[12].argmin())
    assert check(x, d, bad, ua * 0, ud, 9000, 9000, SMP)[:4] == [0, 1, 2, 0]


def test_ends_of_the_uniforms():
    x, d, tok, _, _ = inputs(6, 2, 3000, 3000, F32, 9)
    top = 1.0 - 2.0 ** -24
    for a in (0.0, top):
        for b in (0.0, top):
            ua, ud = torch.full((6, 2), a), torch.full((6,), b)
            acc, out, _ = run(x, d, tok, ua, ud, 3000, 3000, SMP)
            for s in range(6):
                res, _ = oq.verify(x.view(6, 3, -1)[s].numpy(), d.view(6, 2, -1)[s].numpy(), tok[s].tolist(), 2,
                                   ua[s].double().numpy(), b, SMP)
                assert out[s] == res + [-1] * (3 - len(res))


def test_rows_with_nan_still_give_tokens():
    """A NaN counts as absent, so it is neither drawn nor in the way."""
    x, d, tok, ua, ud = inputs(3, 2, 4000, 4000, F32, 10)
    g = torch.Generator().manual_seed(1)
    for a in (x, d):
        a[torch.rand(a.shape, generator=g) < 0.3] = float("nan")
    check(x, d, tok, ua, ud, 4000, 4000, SMP)


def test_replays_of_a_captured_call():
    k = kvr()
    S, T, V = 5, 3, 20000
    x, d, tok, ua, ud = (t.to(DEV) for t in inputs(S, T, V, V, BF, 11))
    ws = torch.empty(k.verify_draft_workspace_size(S, T, V, V, 20), dtype=torch.uint8, device=DEV)
    acc, out, lens = ints([0] * S), torch.zeros((S, T + 1), dtype=torch.int32, device=DEV), ints([50] * S)
    left = ints([0] * S)

    def call():
        k.verify_draft(x, tok, k.Sampler(*SMP), ua, ud, acc, out, draft_logits=d, len_=lens, len_out=left, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    torch.cuda.synchronize()
    for seed in (12, 13, 14):
        for a, b in zip((x, d, tok, ua, ud), inputs(S, T, V, V, BF, seed)):
            a.copy_(b)
        ws.fill_(0xff)
        call()
        torch.cuda.synchronize()
        ref = [t.clone() for t in (acc, out, left)]
        for t in (acc, out, left):
            t.fill_(-5)
        ws.fill_(0)
        torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((acc, out, left), ref))


def test_draft_attend_verify_commit():
    """The operators as a program uses them. A target reads three drafted tokens (and the one before) of four
    sequences over its 4-bit contexts and its own rows in one call; verification cuts the lengths; the tokens that
    stand join the 4-bit context, so that the next call attends to the same tokens from there."""
    k = kvr()
    S, L, Hkv, G, D, T, V = 4, 2, 2, 6, 128, 3, 5000
    g = torch.Generator().manual_seed(20)

    def normal(*shape):
        return torch.randn(shape, generator=g).to(BF).to(DEV)
    lens = [100, 33, 0, 64]
    ctx = k.QuantCache.empty(S, L, Hkv, 200, D)
    base = [normal(S, L, Hkv, 100, D) for _ in range(2)]
    k.quant_append(ctx, ints([0] * S), k.Cache(*base), count=ints(lens))
    own = k.Cache(torch.zeros((S, L, Hkv, 40, D), dtype=BF, device=DEV), torch.zeros((S, L, Hkv, 40, D), dtype=BF, device=DEV))
    cl, ol = ints(lens), ints([T + 1] * S)
    q, kn, vn = normal(S, L, G * Hkv, T + 1, D), normal(S, L, Hkv, T + 1, D), normal(S, L, Hkv, T + 1, D)
    out = torch.empty_like(q)
    ws = torch.empty(k.quant_attn_workspace_size(ctx, own, G * Hkv, T + 1) + 16, dtype=torch.uint8, device=DEV)
    k.quant_attn(ctx, cl, q, out, 0.09, own=own, len_=ol, k_new=kn, v_new=vn, workspace=ws)
    x, d, tok, ua, ud = inputs(S, T, V, V, BF, 21)
    acc, toks = ints([0] * S), torch.zeros((S, T + 1), dtype=torch.int32, device=DEV)
    wv = torch.empty(k.verify_draft_workspace_size(S, T, V, V, 20), dtype=torch.uint8, device=DEV)
    k.verify_draft(x.to(DEV), tok.to(DEV), k.Sampler(*SMP), ua.to(DEV), ud.to(DEV), acc, toks, draft_logits=d.to(DEV),
                   len_=ol, len_out=ol, workspace=wv)
    # The rows of the tokens that stand (and of the one before them) move to the context.
    k.quant_append(ctx, cl, own, count=ol)
    cl += ol
    held = ol.clone()
    ol.zero_()
    # The next token alone, its own cache empty but for it.
    q1, k1, v1 = normal(S, L, G * Hkv, 1, D), normal(S, L, Hkv, 1, D), normal(S, L, Hkv, 1, D)
    ol += 1
    out1 = torch.empty_like(q1)
    k.quant_attn(ctx, cl, q1, out1, 0.09, own=own, len_=ol, k_new=k1, v_new=v1, workspace=ws)
    torch.cuda.synchronize()
    say("accepted", acc.tolist(), "held", held.tolist())
    for s in range(S):
        res, _ = oq.verify(x.float().numpy().reshape(S, T + 1, V)[s], d.float().numpy().reshape(S, T, V)[s],
                           tok[s].tolist(), T, ua[s].double().numpy(), float(ud[s]), SMP)
        assert toks[s].tolist() == res + [-1] * (T + 1 - len(res)) and held[s] == len(res)
        m = len(res)
        for l in range(L):
            for h in range(Hkv):
                hs = slice(h * G, (h + 1) * G)

                def f(t):
                    return t[s, l, h].double().cpu().numpy()
                ck, cv = (oq.stand_for(b[s, l, h, :lens[s]].float().cpu().numpy(), 32) for b in base)
                for o, qq, kk, vv in (
                        (out, q, np.concatenate([ck, f(kn)]), np.concatenate([cv, f(vn)])),
                        (out1, q1, np.concatenate([ck, oq.stand_for(f(kn)[:m], 32), f(k1)]),
                         np.concatenate([cv, oq.stand_for(f(vn)[:m], 32), f(v1)]))):
                    ref = oq.attend(kk, vv, qq[s, l, hs].double().cpu().numpy(), 0.09)
                    err = np.abs(o[s, l, hs].double().cpu().numpy() - ref)
                    assert (err <= 2.0 ** -8 * np.abs(ref) + 8 * 2.0 ** -11 * np.abs(vv).max()).all()
