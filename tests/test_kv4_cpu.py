"""The 4-bit cache's plain forms against hand-made rows, and what its entry points refuse; no GPU is touched."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest

from tests import kv4_plain as plain

ARG, SHAPE = -1, -2
P = 1 << 20          # a pointer that no refused call follows


def test_plain_codes_on_hand_made_rows():
    # range 15, step 1: borders at the halves, half to even; a tiny offset from a border decides it
    x = np.array([0.0, 0.5, 1.5, 2.5, 7.4, 14.6, 15.0, 3.0])
    code, s, m = plain.quantise(x)
    assert s == 1 and m == 0 and code.tolist() == [0, 0, 2, 2, 7, 15, 15, 3]
    code, s, m = plain.quantise(np.array([-7.5, 7.5, 1e-9, -1e-9, 0.0]))
    assert s == 1 and m == -7.5 and code.tolist() == [0, 15, 8, 7, 8]
    code, s, m = plain.quantise(np.full(4, 3.25))
    assert s == 0 and m == 3.25 and not code.any()
    for bad in ([0.0, np.inf], [np.nan, 1.0], [-3e38, 3e38]):
        assert np.isnan(plain.values(np.array(bad))).all()


def test_plain_bf16_rounding():
    one, step = np.float32(1.0), np.float32(2.0 ** -7)
    assert plain.bf16_round(one + step / 2) == 1.0 and plain.bf16_round(one + 3 * step / 2) == 1 + 2 * step
    assert plain.bf16_round(np.float32(3.0e-40)) != 0


def test_a_fifteenth_by_one_correction_is_the_rounded_quotient():
    # the store's q + (x - 15 q) / 15, with 1 / 15 rounded, for every mantissa; 64 bits hold each step before its rounding: the rest
    # is a few units of q's last place, its product with 24 bits ends 27 places below
    x = np.arange(2 ** 23, 2 ** 24, dtype=np.float64)
    r = np.float64(np.float32(1) / np.float32(15))
    q = (x * r).astype(np.float32).astype(np.float64)
    rest = (x - 15 * q).astype(np.float32).astype(np.float64)
    got = (q + rest * r).astype(np.float32)
    assert np.array_equal(got, x.astype(np.float32) / np.float32(15))


def test_plain_keep():
    w = [1.0, 5.0, 5.0, float("nan"), 2.0, 0.0]
    assert plain.keep(w, range(6), 6, 3, 0, 99) == [4, 1, 2]
    assert plain.keep(w, range(6), 6, 2, 0, 99) == [2, 1]
    assert plain.keep(w, range(6), 6, 3, 1, 5) == [0, 1, 5]
    assert plain.keep(w, range(6), 2, 3, 0, 99) == [0, 1]
    assert plain.keep(w, range(6), 6, 5, 0, 99) == [0, 1, 2, 5, 4]


def _cache(slots=2, heads=4, dh=128, cap=100, data=P):
    from paper_2509_25188_b200 import binding as b
    return b, b.Kv4(data, slots, heads, dh, cap)


def test_bytes_of_a_cache():
    b, _ = _cache()
    n = b.lib.l2pd_kv4_bytes
    assert n(1, 1, 128, 64) == 64 * 136 and n(1, 1, 64, 64) == 64 * 72
    assert n(2, 4, 128, 65) == 2 * 4 * 96 * 136
    assert n(100, 32, 128, 131072) == 100 * 32 * 131072 * 136          # past 32 bits
    for bad in ((0, 1, 128, 1), (1, 0, 128, 1), (1, 1, 96, 1), (1, 1, 128, 0), (-1, 1, 64, 4), (2 ** 31 - 1, 65535, 128, 2 ** 31 - 1)):
        assert n(*bad) == 0


def test_largest_capacity():
    # rounded up to the tiles of 128 keys that attention takes, a sequence has to fit 31 bits
    b, _ = _cache()
    assert b.lib.l2pd_kv4_bytes(1, 1, 64, 2 ** 31 - 128) == (2 ** 31 - 128) * 72 and b.lib.l2pd_kv4_bytes(1, 1, 64, 2 ** 31 - 127) == 0
    assert _store(b, b.Kv4(P, 1, 1, 64, 2 ** 31 - 64)) == SHAPE


def _store(b, c, **kw):
    a = dict(k=P, v=P, B=1, rows=1, ks=512, vs=512)
    a.update(kw)
    return b.lib.l2pd_kv4_store(None, C.byref(c) if c is not None else None, a["k"], a["v"], a["B"], a["rows"], None, None, None, a["ks"], a["vs"])


@pytest.mark.parametrize("kw,status", [(dict(k=None), ARG), (dict(v=None), ARG), (dict(ks=511), SHAPE), (dict(vs=508), SHAPE), (dict(ks=516), SHAPE),
                                       (dict(k=P + 8), SHAPE), (dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(rows=-1), SHAPE),
                                       (dict(B=65535, rows=65535), SHAPE), (dict(B=0), 0), (dict(rows=0, k=None), 0)])
def test_store_refusals(kw, status):
    b, c = _cache()
    assert _store(b, c, **kw) == status
    if status:
        assert b.lib.l2pd_last_error(None).startswith(b"l2pd_kv4_store")


@pytest.mark.parametrize("kw,status", [(dict(data=None), ARG), (dict(data=P + 4), ARG), (dict(dh=32), SHAPE), (dict(heads=0), SHAPE), (dict(cap=0), SHAPE)])
def test_cache_refusals(kw, status):
    b, c = _cache(**kw)
    assert _store(b, c) == status
    assert b.lib.l2pd_kv4_load(None, C.byref(c), 0, P, P, 1, 1, None, None, None, 512, 512) == status
    assert _store(b, None) == ARG


def test_load_refusals():
    b, c = _cache()
    call = lambda dtype=0, k=P, ks=512: b.lib.l2pd_kv4_load(None, C.byref(c), dtype, k, P, 1, 1, None, None, None, ks, 512)
    assert call(dtype=2) == ARG and call(k=None) == ARG and call(ks=504) == SHAPE and call(k=P + 2) == SHAPE


@pytest.mark.parametrize("kw,status", [(dict(q=None), ARG), (dict(out=None), ARG), (dict(lens=None), ARG), (dict(scratch=None), ARG), (dict(hq=6), SHAPE),
                                       (dict(hq=0), SHAPE), (dict(max_len=-1), SHAPE), (dict(qs=1016), SHAPE), (dict(qs=1028), SHAPE),
                                       (dict(os=1020), SHAPE), (dict(q=P + 8), SHAPE), (dict(out=P + 8), SHAPE), (dict(scratch=P + 4), SHAPE),
                                       (dict(nbytes=64), SHAPE), (dict(B=0), 0), (dict(rows=0), 0)])
def test_attention_refusals(kw, status):
    b, c = _cache()
    a = dict(q=P, out=P, lens=P, scratch=P, hq=8, max_len=100, qs=1024, os=1024, B=2, rows=3, nbytes=1 << 30)
    a.update(kw)
    assert b.lib.l2pd_attention_kv4(None, C.byref(c), a["q"], a["out"], None, a["B"], a["rows"], None, None, a["lens"], a["max_len"], a["hq"],
                                    a["qs"], a["os"], 0.1, a["scratch"], a["nbytes"], 0) == status
    if status and a["hq"] == 8 and a["max_len"] >= 0:
        assert b.lib.l2pd_attention_kv4_scratch_bytes(C.byref(c), 2, 3, 8, 100) > 64


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_a_length_beyond_the_capacity_plans_for_the_capacity(rows):
    # partial results for as many CTAs as the capacity's tiles keep busy: 2^31 - 1 passed 32 bits in the count of tiles, and one CTA was left
    b, c = _cache(slots=8, heads=8, cap=5000)
    n = lambda max_len: b.lib.l2pd_attention_kv4_scratch_bytes(C.byref(c), 8, rows, 8, max_len)
    assert n(2 ** 31 - 1) == n(2 ** 31 - 100) == n(5001) == n(5000) > n(40)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_scales_that_are_not_finite(scale):
    # one kernel gave NaN for them, the other took them for 0
    b, c = _cache()
    assert b.lib.l2pd_attention_kv4(None, C.byref(c), P, P, None, 2, 3, None, None, P, 100, 8, 1024, 1024, scale, P, 1 << 30, 0) == ARG
    assert b.lib.l2pd_last_error(None) == b"l2pd_attention_kv4: a finite scale"
    assert b.lib.l2pd_kv4_weights(None, C.byref(c), P, P, P, P, 1, 1, None, None, P, 5, 8, 1024, scale) == ARG
    assert b.lib.l2pd_last_error(None) == b"l2pd_kv4_weights: a finite scale"


def test_ctas_of_single_tokens_fit_an_sm():
    # two partial results of eight columns for each CTA: four CTAs an SM for heads of 64, three for heads of 128, whose shared memory
    # holds no more
    n = {}
    for dh in (64, 128):
        b, c = _cache(slots=64, heads=8, dh=dh, cap=8000)
        n[dh] = b.lib.l2pd_attention_kv4_scratch_bytes(C.byref(c), 64, 1, 32, 8000) // (2 * 8 * (dh + 4) * 4)
    assert n[64] % 4 == 0 and n[128] == n[64] // 4 * 3


def test_scratch_of_batches_that_are_refused():
    b, c = _cache(slots=8, heads=2, cap=5000)
    n = lambda rows, hq: b.lib.l2pd_attention_kv4_scratch_bytes(C.byref(c), 8, rows, hq, 5000)
    assert n(2 ** 30, 2) > 0 and n(2 ** 30, 4) == n(2 ** 31 - 1, 6) == n(2 ** 31 - 1, 16) == n(3, 3) == 0


@pytest.mark.parametrize("kw,status", [(dict(q=None), ARG), (dict(lse=None), ARG), (dict(w=None), ARG), (dict(o=None), ARG), (dict(hq=7), SHAPE),
                                       (dict(qs=8), SHAPE), (dict(B=0), 0), (dict(max_len=0), 0)])
def test_weights_refusals(kw, status):
    b, c = _cache()
    a = dict(q=P, lse=P, w=P, o=P, hq=8, qs=1024, B=1, max_len=5)
    a.update(kw)
    assert b.lib.l2pd_kv4_weights(None, C.byref(c), a["q"], a["lse"], a["w"], a["o"], a["B"], 1, None, None, P, a["max_len"], a["hq"], a["qs"], 0.1) == status


@pytest.mark.parametrize("kw,status", [(dict(w=None), ARG), (dict(kept=None), ARG), (dict(lo=None), ARG), (dict(lo=2 * P), ARG), (dict(keep=0), SHAPE),
                                       (dict(max_len=-1), SHAPE), (dict(into=(2, 4, 128, 63, 1 << 30)), SHAPE), (dict(into=(2, 3, 128, 100, 1 << 30)), SHAPE),
                                       (dict(into=(2, 4, 64, 100, 1 << 30)), SHAPE), (dict(into=(2, 4, 128, 90, P)), ARG),
                                       (dict(into=(2, 4, 128, 100, P + 4096)), ARG), (dict(into=(2, 4, 128, 64, 1 << 30), wi=P), ARG),
                                       (dict(into=(2, 4, 128, 64, 1 << 30), pi=3 * P), ARG), (dict(B=0), 0)])
def test_evict_refusals(kw, status):
    b, c = _cache()
    a = dict(w=P, wi=None, pi=None, kept=P, lo=4 * P, keep=64, max_len=100, B=1, into=None)
    a.update(kw)
    into = b.Kv4(a["into"][4], *a["into"][:4]) if a["into"] else None
    assert b.lib.l2pd_kv4_evict(None, C.byref(c), C.byref(into) if into else None, a["w"], a["wi"], 3 * P, a["pi"], a["B"], None, 2 * P, a["max_len"],
                                a["keep"], 0, None, a["kept"], a["lo"]) == status


def test_eviction_refuses_what_its_bitmap_cannot_hold():
    b, c = _cache(cap=1 << 20)
    assert b.lib.l2pd_kv4_evict(None, C.byref(c), None, P, None, None, None, 1, None, 2 * P, (1 << 19) + 1, 64, 0, None, P, 4 * P) == SHAPE


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), ARG), (dict(dh=63), SHAPE), (dict(dh=258), SHAPE), (dict(dh=0), SHAPE), (dict(rows=-1), SHAPE),
                                       (dict(hq=-1), SHAPE), (dict(q=None), ARG), (dict(ko=None), ARG), (dict(qs=100), SHAPE), (dict(theta=0.0), ARG),
                                       (dict(theta=float("nan")), ARG), (dict(eps=-1.0), ARG), (dict(qo=P, qos=600), ARG), (dict(rows=0), 0),
                                       (dict(hq=0, hk=0), 0)])
def test_norm_rope_refusals(kw, status):
    b, _ = _cache()
    a = dict(dtype=1, q=P, k=P, qo=2 * P, ko=2 * P, rows=3, hq=4, hk=2, dh=128, qs=512, ks=256, qos=512, kos=256, eps=1e-5, theta=1e4)
    a.update(kw)
    assert b.lib.l2pd_qk_norm_rope(None, a["dtype"], a["q"], a["k"], a["qo"], a["ko"], None, None, None, a["rows"], a["hq"], a["hk"], a["dh"], a["qs"],
                                   a["ks"], a["qos"], a["kos"], a["eps"], a["theta"]) == status


def test_rows_that_a_launch_cannot_count_are_refused():
    # `rows` is a promise, not an array: 2^31 - 1 of them for 65 heads pass the grid's 32 bits
    b, c = _cache(heads=65)
    w = 65 * 128
    assert b.lib.l2pd_kv4_store(None, C.byref(c), P, P, 1, 2 ** 31 - 1, P, None, None, w, w) == SHAPE
    assert b.lib.l2pd_kv4_load(None, C.byref(c), 1, P, P, 1, 2 ** 31 - 1, P, None, None, w, w) == SHAPE


@pytest.mark.parametrize("off", [4, 4 * (2 * 4 * 100 - 1)])
def test_weights_refuse_arrays_that_overlap(off):
    b, c = _cache()
    for i, o in ((P, P + off), (P + off, P)):
        assert b.lib.l2pd_kv4_weights(None, C.byref(c), P, P, i, o, 1, 1, None, None, P, 100, 4, 512, 0.1) == ARG


@pytest.mark.parametrize("then", ["nothing to do", "gemm", "attention", "lm_head", "init"])
def test_a_refusal_is_reported_for_its_own_call_alone(then):
    b, c = _cache()
    assert _store(b, c, k=None) == ARG and b.lib.l2pd_last_error(None) != b""
    if then == "nothing to do":
        assert _store(b, c, B=0) == 0
    elif then == "gemm":
        assert b.lib.l2pd_gemm_bf16(None, None, None, None, 1, 8, 8, 0, 0) == ARG
    elif then == "attention":
        assert b.lib.l2pd_attention_bf16(None, None, None, None, None, 1, 1, 1, 64, 64, 64, 64, 0, 0) == ARG
    elif then == "lm_head":
        assert b.lib.l2pd_lm_head_bf16(None, None, None, None, 1, 8, 8, None, None, None, None, 0) == ARG
    else:
        assert b.lib.l2pd_init(None, None, 0, None) == ARG
    assert b.lib.l2pd_last_error(None) == b""
