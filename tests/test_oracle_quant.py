"""Pins of oracle/quant.py: the 4-bit format on values worked out by hand, its
error bound, and that verified tokens are distributed as the target's."""
import numpy as np
import pytest

from oracle import quant as oq


def test_format_by_hand():
    x = np.zeros((1, 32), np.float32)
    x[0, :16] = np.arange(16) * 0.5 - 2.0      # -2 .. 5.5: scale 0.5, offset -2
    x[0, 16:] = [-2.0, 5.5, -1.76, -1.74, 0.24, 0.26] + [1.0] * 10
    n, s, z = oq.quantise(x, 32)
    assert s[0, 0] == np.float16(0.5) and z[0, 0] == np.float16(-2.0)
    assert n[0, :16].tolist() == list(range(16))
    assert n[0, 16:22].tolist() == [0, 15, 0, 1, 4, 5]
    assert oq.value(n, s, z)[0, :16].tolist() == x[0, :16].tolist()


def test_ties_go_to_the_even_code_and_odd_values_to_finite_ones():
    x = np.zeros((1, 32), np.float32)
    x[0, :4] = [0.0, 15.0, 0.5, 1.5]
    x[0, 4:8] = [2.5, np.nan, 7.0, 7.5]
    n, s, z = oq.quantise(x, 32)
    assert n[0, :8].tolist() == [0, 15, 0, 2, 2, 0, 7, 8]
    y = np.full((1, 32), 3.0, np.float32)
    n, s, z = oq.quantise(y, 32)
    assert s[0, 0] == 0 and oq.value(n, s, z).tolist() == y.tolist()
    w = np.zeros((1, 32), np.float32)
    w[0, 0], w[0, 1] = np.inf, -np.inf
    assert np.isfinite(oq.stand_for(w, 32)).all()
    assert abs(oq.stand_for(w, 32)[0, 0] - 16384) <= 16384 * 2.0 ** -10


@pytest.mark.parametrize("group", [32, 64])
def test_error_is_half_a_step(group):
    x = np.random.default_rng(group).normal(size=(400, 128)).astype(np.float32)
    n, s, z = oq.quantise(x, group)
    err = np.abs(oq.value(n, s, z) - x)
    # Half a step, and at the ends what the float16 roundings of scale and offset cost.
    step = s.astype(np.float64).repeat(group, -1)
    assert (err <= 0.5 * step + 15 * step * 2.0 ** -11 + 4 * 2.0 ** -11 + 1e-6).all()


@pytest.mark.parametrize("lookup", [False, True])
def test_verified_tokens_have_the_targets_distribution(lookup):
    """Summed over the draft's tokens, with u integrated exactly: P(token) = sum_x Q(x) [accept x] + rejected mass
    times the residual's draw."""
    rng = np.random.default_rng(3)
    V, smp = 12, (0.9, 7, 0.93)
    lg, dl = rng.normal(size=V) * 1.5, rng.normal(size=V) * 1.5
    ids, p = oq.distribution(lg, *smp)
    P = dict(zip(ids.tolist(), p.tolist()))
    if lookup:
        Q = {int(ids[1]): 1.0}
    else:
        j, q = oq.distribution(dl, *smp)
        Q = dict(zip(j.tolist(), q.tolist()))
    got = np.zeros(V)
    M = 4000
    us = (np.arange(M) + 0.5) / M
    for x, qx in Q.items():
        lim = min(1.0, P.get(x, 0.0) / qx)   # u below it: x stands
        got[x] += qx * lim
        if lim < 1.0:
            draws = [oq.verify(np.stack([lg, lg]), None if lookup else dl[None], [x], 1, [0.5 * (lim + 1)], u, smp)[0]
                     for u in us]
            assert all(len(d) == 1 for d in draws)
            for d in draws:
                got[d[0]] += qx * (1.0 - lim) / M
    want = np.array([P.get(i, 0.0) for i in range(V)])
    assert np.abs(got - want).max() <= 2.0 / M


def test_all_tokens_stand_and_the_next_comes_from_the_last_row():
    V, smp = 9, (1.0, 9, 1.0)
    lg = np.zeros((3, V))
    lg[0, 4] = lg[1, 2] = lg[2, 7] = 50.0
    assert oq.verify(lg, None, [4, 2], 2, [0.99, 0.99], 0.3, smp)[0] == [4, 2, 7]
    assert oq.verify(lg, None, [4, 3], 2, [0.99, 0.01], 0.3, smp)[0] == [4, 2]
    assert oq.verify(lg, None, [-1, 3], 2, [0.0, 0.0], 0.3, smp)[0] == [4]
    assert oq.verify(lg, None, [1, 1], 0, [0.0, 0.0], 0.3, smp)[0] == [4]


def test_attention_of_the_last_tokens_is_torchs_with_a_shifted_causal_mask():
    import torch
    rng = np.random.default_rng(5)
    for N, nq in ((9, 1), (20, 4), (4, 4)):
        k, v, q = rng.normal(size=(N, 16)), rng.normal(size=(N, 16)), rng.normal(size=(3, nq, 16))
        mask = torch.ones(nq, N, dtype=torch.bool).tril(N - nq)
        t = [torch.from_numpy(x).expand(3, -1, -1) for x in (k, v)]
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q), *t, attn_mask=mask, scale=0.3)
        assert np.abs(oq.attend(k, v, q, 0.3) - want.numpy()).max() <= 1e-13
    # Query tokens before the first token see nothing.
    out = oq.attend(k[:2], v[:2], rng.normal(size=(1, 4, 16)), 0.3)
    assert (out[0, :2] == 0).all() and np.abs(out[0, 2] - v[0]).max() <= 1e-15
