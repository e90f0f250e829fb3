"""Refusals of the 4-bit cache's and the verification's entry points, all made
on the host before anything is enqueued, and their size queries (CPU only)."""
import ctypes

import pytest

from paper_2608_15797_amd import kvr

EINVAL, EUNSUP, EWS = -1, -2, -4
B = ctypes.byref


def qc(**kw):
    d = dict(data=4096, S=4, L=2, Hkv=2, cap=100, D=128, group=32)
    d.update(kw)
    return kvr.c_quant_cache(*(d[k] for k in ("data", "S", "L", "Hkv", "cap", "D", "group")))


def cc(**kw):
    d = dict(k=4096, v=8192, pos=None, S=4, L=2, Hkv=2, cap=50, D=128, dtype=1)
    d.update(kw)
    return kvr.c_cache(*(d[k] for k in ("k", "v", "pos", "S", "L", "Hkv", "cap", "D", "dtype")))


def last():
    return kvr.lib.kvr_last_error().decode()


@pytest.mark.parametrize("D,group,row", [(128, 32, 80), (128, 64, 72), (64, 32, 40), (64, 64, 36)])
def test_cache_bytes(D, group, row):
    # Slots in tiles of 32, K and V rows of `row` bytes.
    assert kvr.lib.kvr_quant_cache_bytes(B(qc(cap=100, D=D, group=group))) == 16 * 128 * 2 * row
    assert kvr.lib.kvr_quant_cache_bytes(B(qc(cap=1, D=D, group=group))) == 16 * 32 * 2 * row
    assert kvr.lib.kvr_quant_cache_bytes(B(qc(S=3000, L=28, cap=131072, D=D, group=group))) == \
        3000 * 56 * 131072 * 2 * row


BAD_QUANT = [(dict(S=0), EINVAL), (dict(L=-1), EINVAL), (dict(Hkv=0), EINVAL), (dict(cap=0), EINVAL),
             (dict(D=96), EUNSUP), (dict(group=16), EUNSUP), (dict(group=128), EUNSUP),
             (dict(data=None), EINVAL), (dict(data=4100), EINVAL), (dict(S=1 << 20, L=1 << 10, Hkv=2), EUNSUP)]


@pytest.mark.parametrize("kw,want", BAD_QUANT)
def test_bad_quant_cache(kw, want):
    c = qc(**kw)
    if "data" not in kw:
        assert kvr.lib.kvr_quant_cache_bytes(B(c)) == 0
        assert kvr.lib.kvr_quant_attn_workspace_size(B(c), None, 1, 4, 1) == 0
    assert kvr.lib.kvr_quant_append(B(c), 16, B(cc()), None, None, None) == want
    assert kvr.lib.kvr_quant_read(B(c), B(cc()), None, 16, None) == want
    assert kvr.lib.kvr_quant_attn(B(c), 16, None, None, 16, 1, 4, 1, 1.0, None, None, None, 16, None, 0, None) == want
    assert last()


@pytest.mark.parametrize("kw,want", [(dict(L=3), EINVAL), (dict(Hkv=1), EINVAL), (dict(D=64), EINVAL),
                                     (dict(S=5), EINVAL), (dict(k=None), EINVAL), (dict(v=24), EINVAL),
                                     (dict(dtype=7), EUNSUP), (dict(cap=0), EINVAL)])
def test_bad_rows(kw, want):
    c = cc(**kw)
    assert kvr.lib.kvr_quant_append(B(qc()), 16, B(c), None, None, None) == want
    assert kvr.lib.kvr_quant_read(B(qc()), B(c), None, 16, None) == want
    assert kvr.lib.kvr_quant_attn(B(qc()), 16, B(c), 16, 16, 1, 4, 1, 1.0, None, None, None, 16, None, 0, None) == want


def test_missing_lengths():
    assert kvr.lib.kvr_quant_append(B(qc()), None, B(cc()), None, None, None) == EINVAL
    assert kvr.lib.kvr_quant_read(B(qc()), B(cc()), None, None, None) == EINVAL


def test_grid_limits():
    big = dict(S=1 << 14, L=1 << 10, Hkv=64, cap=64)
    assert kvr.lib.kvr_quant_append(B(qc(**big)), 16, B(cc(S=1 << 14, L=1 << 10, Hkv=64, cap=64)), None, None,
                                    None) == EUNSUP
    assert kvr.lib.kvr_quant_read(B(qc(**big)), B(cc(S=1 << 14, L=1 << 10, Hkv=64, cap=64)), None, 16, None) == EUNSUP


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 16, 17, 64])
def test_launches_of_more_threads_than_32_bits_are_refused(T, D):
    # A tile of 32 slots takes 2 D threads; T rows touch up to T // 32 + 2 tiles.
    units = -(-2 ** 32 // (2 * D * (T // 32 + 2)))
    c = dict(S=units, L=1, Hkv=1, D=D)
    assert kvr.lib.kvr_quant_append(B(qc(cap=32, **c)), 16, B(cc(cap=T, **c)), None, None, None) == EUNSUP
    units = -(-2 ** 32 // (2 * D * ((T + 31) // 32 + 1)))
    c = dict(S=units, L=1, Hkv=1, D=D)
    assert kvr.lib.kvr_quant_read(B(qc(cap=32, **c)), B(cc(cap=T, **c)), None, 16, None) == EUNSUP
    # Attention: a wave (float32: four) per unit and 16 of its rows.
    for dtype, waves in ((0, 4), (1, 1)):
        blocks = (4 * min(T, 64) + 15) // 16
        own = cc(S=-(-2 ** 26 // (waves * blocks)), L=1, Hkv=1, D=D, dtype=dtype)
        args = (B(qc(S=1, L=1, Hkv=1, D=D)), B(own), dtype, 4, T)
        assert kvr.lib.kvr_quant_attn_workspace_size(*args) == 0 and "grid" in last()
        own.S -= 1
        if dtype:
            assert kvr.lib.kvr_quant_attn_workspace_size(*args) > 0


def test_slots_past_31_bits_are_refused():
    top = 2 ** 31 - 64
    for cap in (top + 1, 2 ** 31 - 1):
        c = qc(S=1, L=1, Hkv=1, cap=cap)
        assert kvr.lib.kvr_quant_cache_bytes(B(c)) == 0 and "2^31" in last()
        assert kvr.lib.kvr_quant_append(B(c), 16, B(cc(S=1, L=1, Hkv=1)), None, None, None) == EUNSUP
    assert kvr.lib.kvr_quant_cache_bytes(B(qc(S=1, L=1, Hkv=1, cap=top))) == (top + 31) // 32 * 32 * 160
    one = dict(S=1, L=1, Hkv=1)
    f = kvr.lib.kvr_quant_attn_workspace_size
    assert f(B(qc(cap=top - 50, **one)), B(cc(cap=50, **one)), 1, 4, 1) > 0
    assert f(B(qc(cap=top - 50, **one)), B(cc(cap=51, **one)), 1, 4, 1) == 0 and "2^31" in last()


def attn(own=None, **kw):
    d = dict(ctx_len=16, len=None, q=16, dtype=1, Hq=4, nq=1, scale=1.0, kn=None, vn=None, pos=None, out=16, ws=None,
             nb=0)
    d.update(kw)
    if own is not None and "len" not in kw:
        d["len"] = 16
    return kvr.lib.kvr_quant_attn(B(qc()), d["ctx_len"], B(own) if own is not None else None, d["len"], d["q"],
                                  d["dtype"], d["Hq"], d["nq"], d["scale"], d["kn"], d["vn"], d["pos"], d["out"],
                                  d["ws"], d["nb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(ctx_len=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q=24), EINVAL),
    (dict(out=8), EINVAL), (dict(dtype=2), EUNSUP), (dict(dtype=0), EINVAL), (dict(Hq=5), EINVAL),
    (dict(Hq=0), EINVAL), (dict(Hq=34), EUNSUP), (dict(nq=0), EINVAL), (dict(nq=65), EUNSUP), (dict(kn=16), EINVAL),
    (dict(vn=16), EINVAL), (dict(kn=16, vn=8), EINVAL), (dict(pos=16), EINVAL), (dict(kn=16, vn=16, pos=16), EINVAL),
    (dict(len=None), EINVAL)])
def test_bad_attention(kw, want):
    assert attn(cc(), **kw) == want, last()


def test_attention_without_own():
    assert attn(None, kn=16, vn=16) == EINVAL
    assert attn(None, len=16) == EINVAL
    assert attn(cc(S=6)) == EINVAL     # not a multiple of 4 contexts


def test_attention_workspace_is_checked():
    own = cc()
    n = kvr.lib.kvr_quant_attn_workspace_size(B(qc()), B(own), 1, 4, 1)
    if n:
        assert attn(own, ws=16, nb=n - 1) == EWS
        assert attn(own) == EWS
        assert attn(own, ws=24, nb=n) == EINVAL


SMP = kvr.c_sampler(0.8, 20, 0.95, 0, 0)


def verify(**kw):
    d = dict(x=16, V=1000, ld=1000, d=16, Vd=900, ldd=900, dtype=1, S=3, T=4, tok=16, nd=None, smp=SMP, dsmp=None,
             ua=16, ud=16, acc=16, out=16, len=None, len_out=None, ws=16, nb=1 << 30)
    d.update(kw)
    return kvr.lib.kvr_verify_draft(d["x"], d["V"], d["ld"], d["d"], d["Vd"], d["ldd"], d["dtype"], d["S"], d["T"],
                                    d["tok"], d["nd"], B(d["smp"]) if d["smp"] else None,
                                    B(d["dsmp"]) if d["dsmp"] else None, d["ua"], d["ud"], d["acc"], d["out"],
                                    d["len"], d["len_out"], d["ws"], d["nb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), EINVAL), (dict(tok=None), EINVAL), (dict(ua=None), EINVAL), (dict(ud=None), EINVAL),
    (dict(acc=None), EINVAL), (dict(out=None), EINVAL), (dict(smp=None), EINVAL), (dict(dtype=3), EUNSUP),
    (dict(S=0), EINVAL), (dict(T=0), EINVAL), (dict(T=33), EUNSUP), (dict(V=0), EINVAL), (dict(Vd=1001), EINVAL),
    (dict(Vd=0), EINVAL), (dict(d=None), EINVAL), (dict(Vd=-1), EINVAL), (dict(ld=999), EINVAL),
    (dict(ldd=899), EINVAL), (dict(len=16), EINVAL), (dict(len_out=16), EINVAL),
    (dict(V=(1 << 30) + 1, ld=1 << 31), EUNSUP), (dict(S=1 << 20), EUNSUP),
    (dict(smp=kvr.c_sampler(0.0, 20, 0.9, 0, 0)), EINVAL), (dict(smp=kvr.c_sampler(1.0, 65, 0.9, 0, 0)), EINVAL),
    (dict(smp=kvr.c_sampler(1.0, 0, 0.9, 0, 0)), EINVAL), (dict(smp=kvr.c_sampler(1.0, 5, 0.0, 0, 0)), EINVAL),
    (dict(smp=kvr.c_sampler(float("inf"), 5, 0.5, 0, 0)), EINVAL),
    (dict(dsmp=kvr.c_sampler(1.0, 5, 1.5, 0, 0)), EINVAL), (dict(ws=None), EWS), (dict(nb=8), EWS),
    (dict(ws=8), EINVAL)])
def test_bad_verification(kw, want):
    assert verify(**kw) == want, last()


def test_verification_workspace():
    f = kvr.lib.kvr_verify_draft_workspace_size
    assert f(3, 4, 1000, 900, 20) > 0
    for bad in ((0, 4, 1000, 900, 20), (3, 0, 1000, 900, 20), (3, 33, 1000, 900, 20), (3, 4, 1000, 1001, 20),
                (3, 4, 1000, 900, 0), (3, 4, 1000, 900, 65)):
        assert f(*bad) == 0
