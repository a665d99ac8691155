"""The operators around the 4-bit cache against their plain forms in 64 bits.

Codes, s and m are defined exactly, so what is stored reads back equal, bit for bit.  Attention: with A the largest sum of
magnitudes |scale| sum_d |q_d| (c s + |m|) of a score, a score is off by at most D = A (dh / 16 + 8) 2^-23 (a product of 16 terms adds
at most 2^-23 of the running magnitude, plus eight roundings around it), so a weight by 2 D relative (numerator and sum), plus 2^-20
for the exponentials and sums.  Probabilities times s are rounded to fp16 (2^-11 relative, or 2^-25 of a number that is at least
2^-1 for some key: 2^-24 a key), the output to bf16 (2^-8).  With R the largest |value| of the head: |out - want| <= 2^-8 |want| +
(2^-11 + 2 D + 2^-20 + keys 2^-24) 2 R, |lse - want| <= D + 2^-20 + 2^-22 |want|.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np
import pytest
import torch

from tests import kv4_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _b():
    from paper_2509_25188_b200 import binding
    return binding


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _rand(seed, *shape, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).to(DEV)


def _np(x):
    return x.double().cpu().numpy()


def _same(got, want):
    got, want = got.float().cpu().numpy(), np.asarray(want, np.float32)
    assert np.array_equal(got, want, equal_nan=True), np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))))[:3]


# ---- store and load ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dh,heads,B,rows,start", [(128, 1, 1, 1, 0), (128, 3, 2, 65, 63), (64, 5, 3, 64, 0), (64, 1, 1, 200, 7), (128, 32, 2, 33, 64)])
def test_store_then_load(dh, heads, B, rows, start):
    b = _b()
    c = b.KvCache4(B, heads, dh, start + rows)
    k, v = _rand(1, B, rows, heads, dh), _rand(2, B, rows, heads, dh, scale=30)
    c.store(k, v, key_start=_i32([start] * B))
    for dt in (torch.float32, torch.bfloat16):
        gk, gv = c.load(rows, key_start=_i32([start] * B), dtype=dt)
        rnd = (lambda x: x) if dt == torch.float32 else plain.bf16_round
        _same(gk, rnd(plain.values32(_np(k))))
        _same(gv, rnd(plain.values32(_np(v))))
    if start:
        assert not c.load(start, dtype=torch.float32)[0].any()          # keys before them: still zero


def _odd_rows(dh):
    rows = np.zeros((12, dh), np.float32)
    rows[0] = 3.25                                                      # no range
    rows[1, :5] = [-7.5, 7.5, 1e-9, -1e-9, 0]                           # beside a border of step 1
    rows[2, 0] = np.inf
    rows[3, 7] = np.nan
    rows[4, :2] = [-3e38, 3e38]                                         # range beyond fp32
    rows[5, :2] = [-1e-40, 1e-40]                                       # subnormal step
    rows[6, :3] = [9.2e-41, 0, 1.8e-40]                                 # step rounds to the smallest subnormal or 0
    rows[7] = np.arange(dh) % 16 * 0.5                                  # all sixteen codes
    rows[8] = (np.arange(dh) % 31) * 0.5                                # many values on borders
    rows[8, -1] = 15.0
    rows[9] = -np.linspace(1, 2, dh)
    rows[10] = 3e38
    rows[11, -1] = -np.inf
    return torch.from_numpy(rows).to(torch.bfloat16)


@pytest.mark.parametrize("dh", [64, 128])
def test_rows_at_the_ends_of_the_range(dh):
    b = _b()
    x = _odd_rows(dh).to(DEV)[:, None]
    c = b.KvCache4(1, 1, dh, 12)
    c.store(x, x)
    gk, gv = c.load(12, dtype=torch.float32)
    _same(gk[0], plain.values32(_np(x)))
    _same(gv[0], plain.values32(_np(x)))


def _exact_codes(row, m, s):
    """Codes of one row in rational arithmetic."""
    out = []
    for x in row:
        t = (Fraction(float(x)) - Fraction(float(m))) / Fraction(float(s))
        low = t.__floor__()
        up = t - low > Fraction(1, 2) or (t - low == Fraction(1, 2) and low % 2)
        out.append(min(15, low + int(up)))
    return out


@pytest.mark.parametrize("tiny", [9.2e-41, 1e-39, 1.0e-38, 1.2e-38, 1e-30, 1e-9])
@pytest.mark.parametrize("dh", [64, 128])
def test_values_beside_a_border(dh, tiny):
    """A subnormal moves a quotient off a border as any other number does: 64 bits lose it beside 8, rational numbers do not."""
    b = _b()
    rows = np.zeros((6, dh), np.float32)
    for i, lo in enumerate((-7.5, -8.5, -6.5)):                         # 0 lies on the borders 7.5, 8.5 and 6.5 of step 1
        rows[2 * i, :5] = [lo, lo + 15, tiny, -tiny, 0]
        rows[2 * i + 1, -4:] = [lo + 15, -tiny, tiny, lo]               # the other end of the row, no zero in its quarter
        rows[2 * i + 1, :dh // 2] = tiny
    x = torch.from_numpy(rows).to(torch.bfloat16)
    assert (x[0, 2] != 0) and (x[0, 3] != 0)
    c = b.KvCache4(1, 1, dh, 6)
    c.store(x.to(DEV)[:, None], x.to(DEV)[:, None])
    gk, gv = c.load(6, dtype=torch.float32)
    for i, row in enumerate(x.float().numpy()):
        m = row.min()
        want = np.array(_exact_codes(row, m, 1.0)) + np.float64(m)      # step 1, few bits: exact
        _same(gk[0, i, 0], want)
        _same(gv[0, i, 0], want)


def test_ragged_batch_into_chosen_slots_and_places():
    b = _b()
    c = b.KvCache4(5, 2, 128, 90)
    starts, slots, at = [0, 3, 3, 40, 41], [4, 0, 2, 1], [0, 5, 60, 89]
    k, v = _rand(3, 50, 2, 128), _rand(4, 50, 2, 128)                   # rows 41.. belong to nobody
    c.store(k, v, key_start=_i32(at), slots=_i32(slots), row_start=_i32(starts), max_rows=37)
    gk, gv = c.load(90, dtype=torch.float32)
    want = np.zeros((2, 5, 90, 2, 128), np.float32)
    for i, s in enumerate(slots):
        for r in range(starts[i], starts[i + 1]):
            key = at[i] + r - starts[i]
            if key < 90:                                                # the third sequence runs past the end
                want[0, s, key], want[1, s, key] = plain.values32(_np(k[r])), plain.values32(_np(v[r]))
    _same(gk, want[0])
    _same(gv, want[1])
    pk, _ = c.load(37, key_start=_i32(at), slots=_i32(slots), row_start=_i32(starts), total_rows=41, dtype=torch.float32)
    for i, s in enumerate(slots):
        for r in range(starts[i], starts[i + 1]):
            key = at[i] + r - starts[i]
            _same(pk[r], want[0, s, key] if key < 90 else np.zeros((2, 128)))


def test_strided_rows_and_slots_that_do_not_exist():
    b = _b()
    c = b.KvCache4(2, 2, 64, 64)
    qkv = _rand(5, 2, 10, 3, 2, 64)                                     # fused rows: q, k, v
    k, v = qkv[:, :, 1], qkv[:, :, 2]
    c.store(k, v, slots=_i32([7, -1]))
    assert not c.data.any()
    c.store(k, v, key_start=_i32([-3, 60]), slots=_i32([1, 0]))
    gk, _ = c.load(64, dtype=torch.float32)
    _same(gk[1, :7], plain.values32(_np(k[0, 3:])))
    _same(gk[0, 60:], plain.values32(_np(k[1, :4])))
    assert not gk[1, 7:].any() and not gk[0, :60].any()
    zk, zv = c.load(3, slots=_i32([9]))
    assert not zk.any() and not zv.any()


# ---- attention ---------------------------------------------------------------------------------------------------------------

def _check_attention(q, k, v, out, lse, scale):
    """One sequence: q [rows, Hq, dh], k, v [keys, heads, dh] as stored (bf16)."""
    kk, vv = plain.values(_np(k)), plain.values(_np(v))
    want, wl, _ = plain.attention(_np(q), kk, vv, scale)
    got, gl = _np(out), _np(lse)
    if k.shape[0] == 0:
        assert (got == 0).all() and (gl == -np.inf).all()
        return
    dh, heads = q.shape[2], k.shape[1]
    group = q.shape[1] // heads
    code, s, m = plain.quantise(_np(k))
    size = code * s + np.abs(m)
    for h in range(q.shape[1]):
        a = abs(scale) * (np.abs(_np(q)[:, h]) @ size[:, h // group].T).max(-1)
        d = a * (dh / 16 + 8) * 2.0 ** -23
        r = np.abs(vv[:, h // group]).max()
        tol = 2.0 ** -8 * np.abs(want[:, h]) + ((2.0 ** -11 + 2 * d + 2.0 ** -20 + k.shape[0] * 2.0 ** -24) * 2 * r)[:, None]
        err = np.abs(got[:, h] - want[:, h])
        assert (err <= tol).all(), (h, float((err / tol).max()))
        el = np.abs(gl[:, h] - wl[:, h])
        assert (el <= d + 2.0 ** -20 + 2.0 ** -22 * np.abs(wl[:, h])).all(), (h, float(el.max()))


def _check_by_key_sizes(out, lse, q, k, v, scale, lost=2.0 ** -23):
    """As _check_attention for heads that are all alike (out [heads, rows, dh], q [rows, dh], k, v [keys, dh]), with errors counted against what
    each key contributes: p_j R_j, R_j the largest |value| of its row alone.  A probability times s, and on the tensor cores the value, is
    rounded to fp16 (2^-12 each, of p_j R_j, and twice that with the sum), a value whose row is 2^8 below the largest of its 32 by 2^-12 at
    most; what is below fp16's numbers by `lost` max p R a key: 2^-25 of the reference's unit, and 15 codes of a step of at most
    R / 7.5, or 2^-25 of 2^5 R."""
    kk, vv, q = plain.values(_np(k)), plain.values(_np(v)), _np(q)
    code, s, m = plain.quantise(_np(k))
    r = np.abs(vv).max(-1)
    x = q @ kk.T * scale
    p = np.exp(x - x.max(-1, keepdims=True))
    wl = np.log(p.sum(-1)) + x.max(-1)
    p /= p.sum(-1, keepdims=True)
    want = p @ vv
    d = abs(scale) * (np.abs(q) @ (code * s + np.abs(m)).T).max(-1) * (q.shape[1] / 16 + 8) * 2.0 ** -23
    tol = 2.0 ** -8 * np.abs(want) + ((2.0 ** -10 + 2 * d + 2.0 ** -19) * (p @ r) + len(r) * lost * (p * r).max(-1))[:, None]
    err = np.abs(_np(out) - want)
    assert (err <= tol).all(), float((err / tol).max())
    assert (np.abs(_np(lse) - wl) <= d + 2.0 ** -20 + 2.0 ** -22 * np.abs(wl)).all()


# (heads, group, dh, rows of each sequence, keys of each sequence)
ATTENTION = [
    (1, 1, 128, [1], [1]),
    (1, 1, 64, [1], [2]),
    (2, 4, 128, [1, 1, 1], [63, 64, 65]),
    (8, 4, 128, [1], [1000]),
    (3, 1, 64, [5, 1, 0, 2], [129, 0, 17, 4097]),
    (2, 3, 128, [3, 2], [500, 77]),                    # nine columns: two groups of eight
    (4, 1, 128, [32, 32], [512, 300]),
    (1, 8, 64, [4, 1], [700, 3]),
    (2, 2, 128, [17, 33, 5], [640, 1, 100]),           # more columns than a chunk of 32
    (1, 5, 64, [64], [900]),
    (2, 4, 128, [32, 31], [257, 2000]),                # a block with grouped heads
    (1, 16, 128, [9], [130]),
    (1, 1, 128, [1], [70000]),                         # one long sequence over every SM
    (1, 4, 64, [32], [9000]),
    (2, 8, 128, [40], [1500]),
]


@pytest.mark.parametrize("heads,group,dh,rows,keys", ATTENTION)
def test_attention(heads, group, dh, rows, keys):
    b = _b()
    B, cap = len(rows), max(keys) + 70
    c = b.KvCache4(B + 1, heads, dh, cap)
    n = sum(rows)
    starts = np.concatenate(([0], np.cumsum(rows))).tolist()
    slots = [(i + 1) % (B + 1) for i in range(B)]
    k, v = _rand(6, B, cap, heads, dh, scale=2), _rand(7, B, cap, heads, dh)
    for i, x in enumerate(keys):
        k[i, x:], v[i, x:] = float("nan"), float("inf")                 # behind the end: never read
    c.store(k, v, slots=_i32(slots))
    q = _rand(8, n + 3, heads * group, dh)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    c.attention(q, _i32(keys), max(keys), row_start=_i32(starts), max_rows=max(rows), slots=_i32(slots), out=out, lse=lse, check=True)
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    for i in range(B):
        lo, hi = starts[i], starts[i + 1]
        _check_attention(q[lo:hi], k[i, :keys[i]], v[i, :keys[i]], out[lo:hi], lse[lo:hi], dh ** -0.5)
    o2, l2 = c.attention(q[:n], _i32(keys), cap, row_start=_i32(starts), max_rows=max(rows), slots=_i32(slots))
    for i in range(B):                                                  # another max_len may split otherwise
        lo, hi = starts[i], starts[i + 1]
        _check_attention(q[lo:hi], k[i, :keys[i]], v[i, :keys[i]], o2[lo:hi], l2[lo:hi], dh ** -0.5)
    o3, l3 = c.attention(q[:n], _i32(keys), cap, row_start=_i32(starts), max_rows=max(rows), slots=_i32(slots))
    assert torch.equal(o2, o3) and torch.equal(l2, l3)


@pytest.mark.parametrize("vscale", [1e-30, 1e-6, 1e6, 1e25])
@pytest.mark.parametrize("qscale,rows", [(1e-20, 3), (30.0, 3), (1.0, 40)])
def test_attention_whatever_the_magnitudes(vscale, qscale, rows):
    b = _b()
    c = b.KvCache4(1, 2, 128, 400)
    k, v = _rand(9, 400, 2, 128), _rand(10, 400, 2, 128, scale=vscale)
    v[::7] *= 1e-3                                                      # scales that differ from key to key
    v[5] = float(v[6, 0, 0])                                            # a value row without a range
    q = _rand(11, rows, 2, 128, scale=qscale)
    c.store(k, v)
    out, lse = c.attention(q, _i32([400]), 400)
    _check_attention(q, k, v, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("vscale", [1e32, 1e34, 1e36, 3e37])
@pytest.mark.parametrize("rows,dh", [(1, 128), (12, 64), (30, 128), (40, 64), (70, 128)])
def test_values_near_the_end_of_the_range(rows, dh, vscale):
    b = _b()
    c = b.KvCache4(1, 1, dh, 600)
    k, v, q = _rand(151, 600, 1, dh), _rand(152, 600, 1, dh, scale=vscale), _rand(153, rows, 1, dh)
    v[:40] *= 2.0 ** -100
    c.store(k, v)
    out, lse = c.attention(q, _i32([600]), 600)
    assert out.isfinite().all()
    _check_attention(q, k, v, out, lse, dh ** -0.5)


@pytest.mark.parametrize("rows", [2, 20, 40])
def test_rising_scores_move_the_reference(rows):
    b = _b()
    c = b.KvCache4(1, 1, 128, 1000)
    k, v = _rand(12, 1000, 1, 128, scale=0.1), _rand(13, 1000, 1, 128)
    k[:, 0, :4] += torch.linspace(-20, 20, 1000, device=DEV)[:, None].to(torch.bfloat16)
    q = _rand(14, rows, 1, 128)
    q[:, 0, :4] = 3 * (1 - 2 * (torch.arange(rows, device=DEV) % 2)[:, None]).to(torch.bfloat16)     # rising in even rows, falling in odd ones
    c.store(k, v)
    out, lse = c.attention(q, _i32([1000]), 1000, scale=0.7)
    _check_attention(q, k, v, out, lse, 0.7)


@pytest.mark.parametrize("where", [[0], [16], [31], [9, 3, 20]])
@pytest.mark.parametrize("up", [12, 18, 24, 40])
@pytest.mark.parametrize("rows,dh", [(2, 128), (12, 64), (20, 128), (40, 128), (40, 64), (130, 128)])
def test_large_values_without_weight_leave_the_others(rows, dh, up, where):
    """32 rows of values 2^up larger that receive next to no weight, at the start, in the middle and at the end.  So many heads (all alike)
    that a warp meets several tiles of one."""
    b = _b()
    B, heads, n = 8, 32, 1010
    c = b.KvCache4(B, heads, dh, n)
    k, v = _rand(101, n, dh), _rand(102, n, dh)
    q = _rand(103, rows, dh)
    q[:, :8] = 4
    k[:, :8] = 0.5
    for i, g in enumerate(where):
        v[32 * g:32 * g + 32] *= 2.0 ** (up + 3 * i)
        k[32 * g:32 * g + 32, :8] = -16
    alike = lambda x: x[None, :, None].expand(B, -1, heads, -1).contiguous()
    c.store(alike(k), alike(v))
    out, lse = c.attention(alike(q), _i32([n] * B), n, scale=0.125)     # 66 below the others: 2^-95
    _check_by_key_sizes(out.transpose(1, 2).reshape(B * heads, rows, dh), lse.transpose(1, 2).reshape(B * heads, rows), q, k, v, 0.125)


@pytest.mark.parametrize("up", [7, 8, 9, 12, 14, 20, 40, 90])
@pytest.mark.parametrize("rows,dh", [(20, 128), (33, 128), (40, 64), (70, 64), (130, 128)])
def test_one_large_row_beside_others(rows, dh, up):
    """As above with one row of values in 32 larger, at other places in each 32, and rows of zeros, and values that fall off by 2^20 within 32;
    and with one key in 32 larger."""
    b = _b()
    n = 700
    c = b.KvCache4(1, 1, dh, n)
    k, v = _rand(111, n, dh), _rand(112, n, dh)
    q = _rand(113, rows, dh)
    q[:, :8] = 4
    k[:, :8] = 0.5
    large = torch.arange(0, n, 37, device=DEV)
    v[large] *= 2.0 ** up
    k[large, :8] = -16
    v[5:640:64] = 0
    v[320:352] *= (2.0 ** -(torch.arange(32, device=DEV) * 0.7).float())[:, None].to(torch.bfloat16)
    c.store(k[:, None], v[:, None])
    out, lse = c.attention(q[:, None], _i32([n]), n, scale=0.125)
    _check_by_key_sizes(out.transpose(0, 1), lse.transpose(0, 1), q, k, v, 0.125)
    # scores are counted against each key's own size: a key without weight has no part in the others' error
    v = _rand(114, n, dh)
    k[large] = _rand(115, len(large), dh) * 0.01
    k[large, :8] = -1
    k[large] *= 2.0 ** min(up, 60)
    c.store(k[:, None], v[:, None])
    out, lse = c.attention(q[:, None], _i32([n]), n, scale=0.125)
    few = torch.ones(n, dtype=torch.bool, device=DEV)
    few[large] = False
    _check_by_key_sizes(out.transpose(0, 1), lse.transpose(0, 1), q, k[few], v[few], 0.125)     # the large ones' scores: -512 and less


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("rows,dh", [(2, 128), (12, 64), (20, 128), (40, 128), (40, 64), (130, 128)])
def test_values_that_grow_as_their_weights_fall(rows, dh, order):
    """From group to group of 32 keys the values are eight times larger and the weights about eight times smaller, 2^93 in all, or the other
    way round: every group counts."""
    b = _b()
    B, heads, n = 8, 32, 1024
    c = b.KvCache4(B, heads, dh, n)
    k, v = _rand(104, n, dh, scale=0.2), _rand(105, n, dh)
    q = _rand(106, rows, dh, scale=0.2)
    q[:, :8] = 4
    step = torch.arange(n, device=DEV) // 32
    step = step if order > 0 else 31 - step
    v = (v.float() * (2.0 ** (3.0 * step - 50))[:, None]).to(torch.bfloat16)
    k[:, :8] = (-step * np.log(8) / (32 * 0.125))[:, None].to(torch.bfloat16)
    alike = lambda x: x[None, :, None].expand(B, -1, heads, -1).contiguous()
    c.store(alike(k), alike(v))
    out, lse = c.attention(alike(q), _i32([n] * B), n, scale=0.125)
    _check_by_key_sizes(out.transpose(1, 2).reshape(B * heads, rows, dh), lse.transpose(1, 2).reshape(B * heads, rows), q, k, v, 0.125)


@pytest.mark.parametrize("rows", [2, 12, 20])
def test_scores_beyond_24_bits_beside_growing_values(rows):
    """One key leads by millions for every row, where a reference no longer moves by small steps: its value comes out as it is."""
    b = _b()
    B, heads, n, dh = 8, 32, 1024, 128
    c = b.KvCache4(B, heads, dh, n)
    k, v = _rand(107, n, dh), _rand(108, n, dh)
    v[512:] *= 2.0 ** 30
    best = 100 + torch.arange(rows, device=DEV)
    q = k[best] * 2.0 ** 22
    alike = lambda x: x[None, :, None].expand(B, -1, heads, -1).contiguous()
    c.store(alike(k), alike(v))
    out, _ = c.attention(alike(q), _i32([n] * B), n, scale=1.0)
    want = plain.values(_np(v[best]))
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(want).max(-1, keepdims=True)
    assert (np.abs(_np(out.transpose(1, 2).reshape(B * heads, rows, dh)) - want) <= tol).all()


@pytest.mark.parametrize("power", [16, 22, 40])
@pytest.mark.parametrize("rows,dh", [(2, 128), (20, 64), (33, 128), (40, 64), (40, 128), (130, 128), (130, 64)])
def test_scores_of_millions(rows, dh, power):
    """Every third row of queries is 2^power larger: one key leads by far there and its value comes out as it is; other rows as ever."""
    b = _b()
    B, heads, n = 8, 32, 1024
    c = b.KvCache4(B, heads, dh, n)
    k, v = _rand(131, n, dh), _rand(132, n, dh)
    v[512:] *= 2.0 ** 6
    best = 700 - torch.arange(rows, device=DEV)
    q = k[best] * 0.125
    q[::3] *= 2.0 ** power
    alike = lambda x: x[None, :, None].expand(B, -1, heads, -1).contiguous()
    c.store(alike(k), alike(v))
    out, lse = c.attention(alike(q), _i32([n] * B), n, scale=1.0)
    out, lse = out.transpose(1, 2).reshape(B * heads, rows, dh), lse.transpose(1, 2).reshape(B * heads, rows)
    want = plain.values(_np(v[best[::3]]))
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(want).max(-1, keepdims=True)
    assert (np.abs(_np(out[:, ::3]) - want) <= tol).all()
    others = torch.arange(rows, device=DEV) % 3 != 0
    _check_by_key_sizes(out[:, others], lse[:, others], q[others], k, v, 1.0)


@pytest.mark.parametrize("less", [15.0, 24.0, 26.0])
@pytest.mark.parametrize("rows,dh", [(2, 128), (12, 64), (20, 128), (40, 128), (40, 64), (130, 128)])
def test_many_small_weights_beside_a_large_one(rows, dh, less):
    """The first key leads by 2^less, and has no part in half of the dimensions: what is there comes from a thousand small weights."""
    b = _b()
    B, heads, n = 8, 32, 1024
    c = b.KvCache4(B, heads, dh, n)
    k, v = _rand(141, n, dh, scale=0.05), _rand(142, n, dh) + 1
    k[:, 0] = 0
    k[0] = 0
    k[0, 0] = 2
    v[0, :dh // 2], v[0, dh // 2:] = 0, 1                               # code 0 of 0: exactly nothing
    q = _rand(143, rows, dh, scale=0.1)
    q[:, 0] = float(np.float32(less * np.log(2) / 2))
    alike = lambda x: x[None, :, None].expand(B, -1, heads, -1).contiguous()
    c.store(alike(k), alike(v))
    out, _ = c.attention(alike(q), _i32([n] * B), n, scale=1.0)
    got = _np(out.transpose(1, 2).reshape(B * heads, rows, dh))[..., :dh // 2]
    kk, vv, q = plain.values(_np(k)), plain.values(_np(v)), _np(q)
    code, s, m = plain.quantise(_np(k))
    x = q @ kk.T
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    want, r = (p @ vv)[:, :dh // 2], np.abs(vv).max(-1)
    d = (np.abs(q) @ (code * s + np.abs(m)).T).max(-1) * (dh / 16 + 8) * 2.0 ** -23
    # as in _check_by_key_sizes, over the keys that count here; 2^-25 of fp16 is 2^-34 of the largest
    tol = 2.0 ** -8 * np.abs(want) + ((2.0 ** -10 + 2 * d + 2.0 ** -19) * (p[:, 1:] @ r[1:]) + n * 2.0 ** -32 * (p * r).max(-1))[:, None]
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
@pytest.mark.parametrize("rows", [2, 12, 20, 40, 130])
def test_any_scale_and_ragged_last_tiles(rows, scale, dh):
    b = _b()
    c = b.KvCache4(2, 1, dh, 300)
    k, v = _rand(41, 2, 300, 1, dh), _rand(42, 2, 300, 1, dh)
    k[:, 200:], v[:, 200:] = float("nan"), float("nan")
    k[0, 64:96] = 0                                                     # a group of keys, and one of values, without magnitude
    v[0, 32:64] = 0
    v[1, :33] = 0
    q = _rand(43, 2, rows, 1, dh)
    c.store(k, v)
    lens = [131, 33]
    out, lse = c.attention(q, _i32(lens), 300, scale=scale)
    for i, n in enumerate(lens):
        _check_attention(q[i], k[i, :n], v[i, :n], out[i], lse[i], scale)


def _uneven_queries(rows, dh):
    """Keys without negative numbers, 0 in dimension 0 of every one (kept exactly), and a block of queries whose row 1 is 2^60 in that dimension
    alone: its scores are 0, and the other rows' are what they would be without it."""
    b = _b()
    c = b.KvCache4(1, 1, dh, 500)
    k, v = _rand(91, 500, 1, dh).abs(), _rand(92, 500, 1, dh)
    k[..., 0] = 0
    q = _rand(93, rows, 1, dh, scale=3)
    q[1] = 0
    q[1, 0, 0] = 2.0 ** 60
    q[rows // 2 + 1 if rows > 2 else 0] *= 2.0 ** -10
    c.store(k, v)
    return b, c, k, v, q


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rows", [2, 3, 12, 20, 40, 130])
def test_a_row_does_not_decide_the_precision_of_others(rows, dh):
    b, c, k, v, q = _uneven_queries(rows, dh)
    n = _i32([500])
    out, lse = c.attention(q, n, 500)
    _check_attention(q, k, v, out, lse, dh ** -0.5)
    w = c.attention_weights(q, lse, n, 500, torch.zeros(1, 1, 500, device=DEV))
    kk, qn = plain.values(_np(k)), _np(q)
    _, _, want = plain.attention(qn, kk, kk, dh ** -0.5)
    code, s, m = plain.quantise(_np(k))
    d = (np.abs(qn[:, 0]) @ (code * s + np.abs(m))[:, 0].T).max() * dh ** -0.5 * (dh / 16 + 8) * 2.0 ** -23     # as in test_weights
    assert (np.abs(_np(w)[0] - want) <= (2 * d + 2.0 ** -19 + rows * 2.0 ** -24) * want + 2.0 ** -23 * want).all()


@pytest.mark.parametrize("rows", [2, 40])
def test_nan_stays_where_it_belongs(rows):
    b = _b()
    c = b.KvCache4(1, 3, 64, 200)
    k, v, q = _rand(15, 200, 3, 64), _rand(16, 200, 3, 64), _rand(17, rows, 3, 64)
    k[150, 0, 3] = float("nan")
    v[20, 1, 60] = float("inf")
    q[1, 2, 5] = float("inf")
    c.store(k, v)
    out, lse = c.attention(q, _i32([200]), 200)
    assert out[:, 0].isnan().all() and lse[:, 0].isnan().all()
    assert out[:, 1].isnan().all() and lse[:, 1].isfinite().all()
    assert out[1, 2].isnan().all() and out[0, 2].isfinite().all()
    w = c.attention_weights(q, lse, _i32([200]), 200, torch.zeros(1, 3, 200, device=DEV))
    assert w[0, 1].isfinite().all() and w[0, 0].isnan().all()
    out, lse = c.attention(q, _i32([150]), 200)                         # the bad key behind the end
    assert out[:, 0].isfinite().all()


def test_cache_past_32_bits():
    b = _b()
    slots, heads, cap = 9, 32, 131072                                   # 5.1 GB
    c = b.KvCache4(slots, heads, 128, cap)
    assert c.data.numel() > 2 ** 32
    k, v, q = _rand(18, 1, 100, heads, 128), _rand(19, 1, 100, heads, 128), _rand(20, 1, 1, heads, 128)
    at, slot = _i32([cap - 100]), _i32([slots - 1])
    c.store(k, v, key_start=at, slots=slot)
    gk, gv = c.load(100, key_start=at, slots=slot, dtype=torch.float32)
    _same(gk, plain.values32(_np(k)))
    _same(gv, plain.values32(_np(v)))
    out, lse = c.attention(q, _i32([cap]), cap, slots=slot)
    kk, vv = np.zeros((cap, 1, 128)), np.zeros((cap, 1, 128))
    kk[-100:], vv[-100:] = plain.values(_np(k[0, :, -1:])), plain.values(_np(v[0, :, -1:]))
    want, wl, ww = plain.attention(_np(q[0, :, -1:]), kk, vv, 128 ** -0.5)
    assert np.abs(_np(out[0, :, -1]) - want[:, 0]).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -11 * np.abs(vv).max() * 100 / cap * 8
    assert np.abs(_np(lse[0, :, -1]) - wl[:, 0]).max() <= 2.0 ** -17
    w = c.attention_weights(q, lse, _i32([cap]), cap, torch.zeros(slots, heads, cap, device=DEV), slots=slot)
    assert not w[:-1].any() and np.abs(_np(w[-1, -1]) - ww[0]).max() <= 2.0 ** -15 * ww.max()


def test_other_streams_captures_and_strides():
    b = _b()
    c = b.KvCache4(2, 2, 128, 300)
    k, v = _rand(21, 2, 300, 2, 128), _rand(22, 2, 300, 2, 128)
    wide = _rand(23, 2, 9, 3, 4, 128)
    q = wide[:, :, 1]                                                   # rows 12 heads apart
    store = torch.zeros(2, 9, 3, 4, 128, dtype=torch.bfloat16, device=DEV)
    out = store[:, :, 2]
    lens = _i32([300, 41])
    c.store(k, v)
    want, wl = c.attention(q.contiguous(), lens, 300)
    lse = torch.empty(2, 9, 4, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.attention(q, lens, 300, out=out, lse=lse)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl) and not store[:, :, :2].any()
    # two graphs over the same cache, replayed in turn and with changed lengths
    outs, graphs = [torch.zeros_like(want) for _ in range(2)], []
    weights = torch.zeros(2, 2, 300, device=DEV)
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _, l = c.attention(q, lens, 300, out=outs[i])
            c.attention_weights(q, l, lens, 300, weights)
        graphs.append(g)
    lens.copy_(_i32([7, 300]))
    for g in (0, 1, 0, 1):
        graphs[g].replay()
    torch.cuda.synchronize()
    again, al = c.attention(q, lens, 300)
    assert torch.equal(outs[0], again) and torch.equal(outs[1], again)
    once = c.attention_weights(q, al, lens, 300, torch.zeros(2, 2, 300, device=DEV))
    assert torch.allclose(weights, 4 * once, rtol=2.0 ** -21, atol=0)   # four additions, a half-ulp each


@pytest.mark.parametrize("rows", [1, 40])
def test_lengths_written_just_before_the_call(rows):
    """The lengths of a call are those the stream holds when it runs, for all of its kernels: they change from call to call, behind a
    store and behind an eviction, with nothing waited for in between."""
    b = _b()
    B, heads, cap = 3, 2, 700
    c, d = b.KvCache4(B, heads, 128, cap), b.KvCache4(B, heads, 128, cap)
    k, v, q = _rand(61, B, cap, heads, 128), _rand(62, B, cap, heads, 128), _rand(63, B, rows, 2 * heads, 128)
    c.store(k, v)
    w = torch.rand(B, heads, cap, generator=torch.Generator().manual_seed(64)).to(DEV)
    plan = [_i32([(131 * i * (j + 1)) % (cap + 1) for j in range(B)]) for i in range(24)]
    lens, got = _i32([0] * B), []
    for i, n in enumerate(plan):
        lens.copy_(n)
        c.store(k, v)
        first = c.attention(q, lens, cap)
        kept, left = c.evict(w, lens, cap, 200 + i, into=d)
        got.append(first + d.attention(q, left, cap))
    torch.cuda.synchronize()
    for i, (n, have) in enumerate(zip(plan, got)):
        one = c.attention(q, n, cap)
        torch.cuda.synchronize()
        _, left = c.evict(w, n, cap, 200 + i, into=d)
        torch.cuda.synchronize()
        want = one + d.attention(q, left, cap)
        assert left.tolist() == [min(x, 200 + i) for x in n.tolist()]
        for x, y in zip(have, want):
            assert torch.equal(x, y), i


def test_calls_at_once_on_two_streams():
    """Attention of both kinds, weights and stores into another cache, on two streams with nothing between them: the bits are those of
    the calls one after the other."""
    b = _b()
    c, other = b.KvCache4(2, 4, 128, 3000), [b.KvCache4(2, 4, 128, 3000) for _ in range(2)]
    k, v = _rand(71, 2, 3000, 4, 128), _rand(72, 2, 3000, 4, 128)
    c.store(k, v)
    lens = _i32([3000, 1234])
    qs = [_rand(73, 2, 5, 8, 128), _rand(74, 2, 50, 8, 128), _rand(75, 2, 16, 8, 128)]
    want = [c.attention(q, lens, 3000) for q in qs]
    sums = [c.attention_weights(q, l, lens, 3000, torch.zeros(2, 4, 3000, device=DEV)) for q, (_, l) in zip(qs, want)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for turn in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                q = (turn + i) % 3
                o, l = c.attention(qs[q], lens, 3000)
                got[i].append((q, o, l, c.attention_weights(qs[q], l, lens, 3000, torch.zeros(2, 4, 3000, device=DEV))))
                other[i].store(k, v)
    for s in streams:
        s.synchronize()
    for q, o, l, w in got[0] + got[1]:
        assert torch.equal(o, want[q][0]) and torch.equal(l, want[q][1]) and torch.equal(w, sums[q])
    for x in other:
        assert torch.equal(x.data, c.data)


@pytest.mark.parametrize("rows,heads,dh", [(130, 32, 128), (130, 32, 64), (128, 8, 128), (64, 32, 128), (40, 32, 128), (32, 32, 128), (9, 32, 64), (1, 32, 128)])
def test_many_calls_give_the_same_bits(rows, heads, dh):
    """Every CTA goes through several pieces and tiles, whose buffers follow one another as fast as they can: 200 calls, all heads alike."""
    b = _b()
    B, n = 8, 1010
    c = b.KvCache4(B, heads, dh, n)
    alike = lambda x: x[None, :, None].expand(B, -1, heads, -1).contiguous()
    c.store(alike(_rand(121, n, dh)), alike(_rand(122, n, dh)))
    q, lens = alike(_rand(123, rows, dh)), _i32([n] * B)
    w = torch.zeros(B, heads, n, device=DEV)
    out, lse = c.attention(q, lens, n)
    once = c.attention_weights(q, lse, lens, n, w, out=torch.empty_like(w))
    differ = torch.zeros(3, dtype=torch.int64, device=DEV)
    for _ in range(200):
        o, l = c.attention(q, lens, n)
        differ += torch.stack([(o != out).sum(), (l != lse).sum(), (c.attention_weights(q, lse, lens, n, w, out=torch.empty_like(w)) != once).sum()])
    assert differ.tolist() == [0, 0, 0]


def test_batches_without_rows():
    b = _b()
    c = b.KvCache4(2, 2, 64, 50)
    c.store(_rand(81, 2, 50, 2, 64), _rand(82, 2, 50, 2, 64))
    before = c.data.clone()
    none, q, lens, start = _rand(83, 0, 2, 64), _rand(84, 0, 4, 64), _i32([50, 9]), _i32([0, 0, 0])
    c.store(none, none, row_start=start, max_rows=5)
    k, v = c.load(5, row_start=start, total_rows=0)
    out, lse = c.attention(q, lens, 50, row_start=start, max_rows=5)
    assert k.shape == v.shape == (0, 2, 64) and out.shape == (0, 4, 64) and lse.shape == (0, 4)
    w = torch.rand(2, 2, 50, device=DEV)
    new = c.attention_weights(q, lse, lens, 50, w, out=torch.full_like(w, -1.0), row_start=start, max_rows=5)
    for i, n in enumerate([50, 9]):
        assert torch.equal(new[i, :, :n], w[i, :, :n]) and (new[i, :, n:] == -1).all()
    assert c.attention(_rand(85, 0, 3, 4, 64), _i32([]), 50)[0].shape == (0, 3, 4, 64)
    assert b.qk_norm_rope(_rand(86, 0, 4, 64), none)[0].shape == (0, 4, 64)
    assert torch.equal(c.data, before)


def test_binding_refuses_wrong_tensors():
    b = _b()
    c = b.KvCache4(1, 2, 128, 10)
    x, n = _rand(24, 5, 2, 128), _i32([5])
    for bad in (x.float(), x[:, :1], x.cpu(), x.transpose(0, 1), x.view(5, 4, 64)):
        with pytest.raises(ValueError):
            c.store(bad, bad)
    with pytest.raises(ValueError):
        c.attention(x, n.long(), 5)
    with pytest.raises(ValueError):
        c.attention(x, n.cpu(), 5)
    with pytest.raises(ValueError):
        c.store(x, x, row_start=_i32([0, 5]))
    with pytest.raises(ValueError):
        c.attention_weights(x, torch.zeros(5, 2, device=DEV), n, 5, torch.zeros(1, 2, 9, device=DEV))
    with pytest.raises(b.L2pdError):
        c.attention(_rand(24, 5, 3, 128), n, 5)                         # three query heads on two key heads
    with pytest.raises(b.L2pdError):
        b.KvCache4(1, 2, 96, 10)


# ---- weights -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,group,dh,rows,keys", [a for a in ATTENTION if max(a[4]) < 10000])
def test_weights(heads, group, dh, rows, keys):
    b = _b()
    B, cap = len(rows), max(keys) + 5
    c = b.KvCache4(B, heads, dh, cap)
    n = sum(rows)
    starts = np.concatenate(([0], np.cumsum(rows))).tolist()
    k, v, q = _rand(25, B, cap, heads, dh), _rand(26, B, cap, heads, dh), _rand(27, n, heads * group, dh)
    c.store(k, v)
    lens, rs = _i32(keys), _i32(starts)
    _, lse = c.attention(q, lens, cap, row_start=rs, max_rows=max(rows))
    base = torch.rand(B, heads, cap, device=DEV)
    out = torch.full_like(base, -1.0)
    c.attention_weights(q, lse, lens, cap, base, out=out, row_start=rs, max_rows=max(rows))
    inplace = base.clone()
    c.attention_weights(q, lse, lens, cap, inplace, row_start=rs, max_rows=max(rows))
    for i in range(B):
        kk = plain.values(_np(k[i, :keys[i]]))
        qi = _np(q[starts[i]:starts[i + 1]])
        _, _, w = plain.attention(qi, kk, kk, dh ** -0.5)
        assert (out[i, :, keys[i]:] == -1).all() and torch.equal(inplace[i, :, keys[i]:], base[i, :, keys[i]:])
        got, was = _np(out[i, :, :keys[i]]), _np(base[i, :, :keys[i]])
        # a weight is off by twice the score's error, relative, plus the exponential's; the sums of rows * group terms by 2^-24 each
        code, s, m = plain.quantise(_np(k[i, :keys[i]]))
        a = max((np.abs(qi[:, h]) @ (code * s + np.abs(m))[:, h // group].T).max() for h in range(heads * group)) if w.size and len(qi) else 0.0
        d = a * dh ** -0.5 * (dh / 16 + 8) * 2.0 ** -23
        tol = (2 * d + 2.0 ** -19 + rows[i] * group * 2.0 ** -24) * w + 2.0 ** -23 * (was + w)
        assert (np.abs(got - was - w) <= tol).all()
        assert torch.equal(inplace[i, :, :keys[i]], out[i, :, :keys[i]])


@pytest.mark.parametrize("B", [33, 64, 65, 300])
@pytest.mark.parametrize("rows,group,dh", [(1, 4, 128), (3, 4, 64), (8, 3, 128), (20, 2, 64), (40, 3, 128)])
@pytest.mark.parametrize("kind", ["equal", "ragged"])
def test_more_sequences_than_a_warp_has_lanes(kind, rows, group, dh, B):
    """Every warp surveys the batch 32 sequences at a time; sequences and their pieces must be found behind the first 32 too."""
    b = _b()
    heads, cap = 2, 330
    c = b.KvCache4(B, heads, dh, cap)
    k, v = _rand(161, B, cap, heads, dh), _rand(162, B, cap, heads, dh)
    c.store(k, v)
    counts = [rows] * B if kind == "equal" else [(rows * (5 * i % 7)) // 6 for i in range(B)]
    keys = [257] * B if kind == "equal" else [0 if i % 9 == 4 else 1 + (i * 97) % cap for i in range(B)]
    slots = [(7 * i + 3) % B for i in range(B)] if B % 7 else list(range(B))[::-1]
    starts = np.concatenate(([0], np.cumsum(counts))).tolist()
    q = _rand(163, starts[-1], heads * group, dh)
    lens, rs, sl = _i32(keys), _i32(starts), _i32(slots)
    out, lse = c.attention(q, lens, cap, row_start=rs, max_rows=rows, slots=sl, check=True)
    base = torch.rand(B, heads, cap, device=DEV)
    w = c.attention_weights(q, lse, lens, cap, base, out=torch.full_like(base, -1.0), row_start=rs, max_rows=rows, slots=sl)
    for i in list(range(0, B, 13)) + [31, 32, 33 % B, 63 % B, B - 2, B - 1]:
        lo, hi, n, s = starts[i], starts[i + 1], keys[i], slots[i]
        assert (w[s, :, n:] == -1).all()
        _, _, ww = plain.attention(_np(q[lo:hi]), plain.values(_np(k[s, :n])), plain.values(_np(v[s, :n])), dh ** -0.5)
        got, was = _np(w[s, :, :n]), _np(base[s, :, :n])
        if hi > lo:
            _check_attention(q[lo:hi], k[s, :n], v[s, :n], out[lo:hi], lse[lo:hi], dh ** -0.5)
        code, step, m = plain.quantise(_np(k[s, :n]))                   # as in test_weights
        a = max((np.abs(_np(q[lo:hi])[:, h]) @ (code * step + np.abs(m))[:, h // group].T).max() for h in range(heads * group)) if hi > lo and n else 0.0
        d = a * dh ** -0.5 * (dh / 16 + 8) * 2.0 ** -23
        assert (np.abs(got - was - ww) <= (2 * d + 2.0 ** -19 + rows * group * 2.0 ** -24) * ww + 2.0 ** -23 * (was + ww)).all()


# ---- eviction ----------------------------------------------------------------------------------------------------------------

def _weights(kind, B, heads, cap):
    g = torch.Generator().manual_seed(31)
    w = torch.rand(B, heads, cap, generator=g)
    if kind == "ties":
        w = torch.round(w * 4) / 4
    elif kind == "equal":
        w = torch.zeros_like(w)
        w[:, :, ::2] = -0.0
    elif kind == "wild":
        w = (w - 0.5) * 10.0 ** torch.randint(-38, 38, w.shape, generator=g)
        w[:, :, 3::11] = float("nan")
        w[:, :, 5::13] = float("inf")
        w[:, :, 7::17] = -float("inf")
    return w.to(DEV)


@pytest.mark.parametrize("into", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "wild"])
@pytest.mark.parametrize("heads,dh,lens,keep,first,guard", [(1, 128, [1], 1, 0, 0), (2, 64, [5, 0, 100, 64], 33, 0, 0), (3, 128, [130, 131], 64, 4, 20),
                                                            (2, 128, [2050, 1500], 1024, 4, 32), (1, 64, [40], 30, 35, 0), (1, 128, [9000], 8999, 0, 1),
                                                            (2, 64, [70000], 1, 0, 0), (1, 128, [70000], 20000, 4, 100)])
def test_evict(into, kind, heads, dh, lens, keep, first, guard):
    b = _b()
    B, cap = len(lens), max(lens) + 3
    slots = list(range(B))[::-1]
    c = b.KvCache4(B, heads, dh, cap)
    k, v = _rand(28, B, cap, heads, dh), _rand(29, B, cap, heads, dh)
    c.store(k, v)
    w = _weights(kind, B, heads, cap)
    pos = torch.arange(cap, dtype=torch.int32, device=DEV).expand(B, heads, cap).contiguous() * 2
    from_ = [2 * max(n - guard, 0) if guard else 2 ** 31 - 1 for n in lens]
    dcap = keep if into else cap
    dst = b.KvCache4(B, heads, dh, dcap) if into else c
    w0, p0, wn = w.clone(), pos.clone(), w.double().cpu().numpy()
    wi = torch.full((B, heads, dcap), -5.0, device=DEV) if into else None
    pi = torch.full((B, heads, dcap), -5, dtype=torch.int32, device=DEV) if into else None
    kept, new = c.evict(w, _i32(lens), max(lens), keep, positions=pos, first=2 * first, protect_from=_i32(from_), slots=_i32(slots),
                        into=dst if into else None, weights_into=wi, positions_into=pi)
    gk, gv = dst.load(dcap, dtype=torch.float32)
    wo, po = (wi, pi) if into else (w, pos)
    assert new.tolist() == [min(n, keep) for n in lens]
    ak, av = plain.values32(_np(k)), plain.values32(_np(v))
    for i, n in enumerate(lens):
        s, m = slots[i], min(lens[i], keep)
        for h in range(heads):
            want = plain.keep(wn[s, h], (2 * np.arange(cap)).tolist(), n, keep, 2 * first, from_[i])
            assert kept[i, h, :m].tolist() == want and (kept[i, h, m:] == -1).all()
            _same(gk[s, :m, h], ak[s, want, h])
            _same(gv[s, :m, h], av[s, want, h])
            assert torch.equal(wo[s, h, :m].view(torch.int32), w0[s, h, want].view(torch.int32)) and torch.equal(po[s, h, :m], p0[s, h, want])
            if into:
                assert (wo[s, h, m:] == -5).all() and (po[s, h, m:] == -5).all() and not gk[s, m:, h].any()
            else:
                assert torch.equal(po[s, h, m:], p0[s, h, m:])
                _same(gk[s, m:, h], ak[s, m:, h])


def test_evict_longer_than_a_cluster_keeps_at_hand():
    b = _b()
    n, keep = 300000, 5000
    c, into = b.KvCache4(1, 1, 64, n), b.KvCache4(1, 1, 64, keep)
    k = _rand(44, 1, n, 1, 64)
    c.store(k, k)
    w = torch.round(torch.rand(1, 1, n, device=DEV) * 64) / 64          # thousands of equal weights at the border
    kept, new = c.evict(w, _i32([n]), n, keep, into=into)
    want = plain.keep(_np(w)[0, 0], range(n), n, keep, 0, 2 ** 31 - 1)
    assert kept[0, 0].tolist() == want and new.tolist() == [keep]
    _same(into.load(keep, dtype=torch.float32)[0][0, :, 0], plain.values32(_np(k[0, want, 0])))


def test_evict_without_positions_and_twice():
    b = _b()
    c = b.KvCache4(1, 2, 128, 600)
    k = _rand(32, 1, 600, 2, 128)
    c.store(k, k)
    w = torch.rand(1, 2, 600, device=DEV)
    wn = _np(w)
    pos = torch.full((1, 2, 600), -1, dtype=torch.int32, device=DEV)
    kept, n1 = c.evict(w, _i32([600]), 600, 300, positions_into=pos)   # no positions yet: an index is its key's position
    first = kept.cpu().numpy()
    assert np.array_equal(pos[0, :, :300].cpu().numpy(), first[0])
    kept, n2 = c.evict(w, n1, 600, 100, positions=pos, protect_from=_i32([590]))
    for h in range(2):
        p1 = first[0, h]
        want = plain.keep(wn[0, h][p1], p1.tolist(), 300, 100, 0, 590)
        assert kept[0, h].tolist() == want and pos[0, h, :100].tolist() == p1[want].tolist()
        _same(c.load(100, dtype=torch.float32)[0][0, :, h], plain.values32(_np(k))[0, p1[want], h])


@pytest.mark.parametrize("keep", [2 ** 31 - 1, 2 ** 31 - 130])
def test_evict_that_keeps_everything(keep):
    """`keep` as "no limit": every key stays, and the places behind them say so to the last one."""
    b = _b()
    c = b.KvCache4(1, 1, 64, 9000)
    k = _rand(45, 1, 9000, 1, 64)
    c.store(k, k)
    before, w = c.data.clone(), torch.rand(1, 1, 9000, device=DEV)
    kept, new = c.evict(w, _i32([8999]), 9000, keep)                    # 8.6 GB of places
    assert new.tolist() == [8999] and kept.shape == (1, 1, keep)
    assert torch.equal(kept[0, 0, :8999], torch.arange(8999, dtype=torch.int32, device=DEV))
    assert int(kept[0, 0, 8999:].max()) == -1 and int(kept[0, 0, 8999:].min()) == -1
    assert torch.equal(c.data, before)
    del kept
    kept, new = c.evict(w, _i32([5]), 0, 7)                             # no key may be read
    assert new.tolist() == [0] and (kept == -1).all()


def test_a_captured_step_of_all_calls():
    """Norm + rotation, store, attention, weights, eviction and load in one graph, replayed on new inputs, against the calls one by one."""
    b = _b()
    B, heads, group, dh, rows, cap, keep = 3, 2, 2, 128, 20, 5000, 1500
    prompt = _rand(171, B, cap - rows, heads, dh), _rand(172, B, cap - rows, heads, dh)
    pos = torch.arange(rows, dtype=torch.int32, device=DEV).repeat(B) + cap
    q, k, v = (_rand(173 + i, B, rows, h, dh) for i, h in enumerate((heads * group, heads, heads)))
    gain = torch.ones(dh, device=DEV)
    start, lens = _i32([cap - rows, 4000, 70]), _i32([cap, 4020, 90])

    def fresh():
        c, d = b.KvCache4(B, heads, dh, cap), b.KvCache4(B, heads, dh, keep)
        c.store(*prompt)
        return c, d, torch.zeros(B, heads, cap, device=DEV), torch.zeros(B, heads, keep, device=DEV)

    def step(c, d, w, wi):
        qr, kr = b.qk_norm_rope(q.view(B * rows, -1, dh), k.view(B * rows, heads, dh), gain, gain, pos)
        c.store(kr.view(k.shape), v, key_start=start)
        out, lse = c.attention(qr.view(q.shape), lens, cap)
        c.attention_weights(qr.view(q.shape), lse, lens, cap, w)
        kept, left = c.evict(w, lens, cap, keep, first=4, into=d, weights_into=wi)
        return (out, lse, kept, left, *d.load(keep, dtype=torch.float32))

    state = fresh()
    step(*state)                                                        # once outside
    for x in (state[0].data, state[1].data, state[2], state[3]):
        x.zero_()
    state[0].store(*prompt)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*state)
    other = fresh()
    for turn in range(3):
        for i, x in enumerate((q, k, v)):
            x.copy_(_rand(181 + 3 * turn + i, *x.shape))
        lens.copy_(_i32([cap - turn, 4020, 90 + turn]))
        graph.replay()
        want = step(*other)
        torch.cuda.synchronize()
        for x, y in zip(got + (state[2], state[3], state[0].data, state[1].data), want + (other[2], other[3], other[0].data, other[1].data)):
            assert torch.equal(x, y), turn


# ---- norms and rotation ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype,rows,hq,hk,dh,start", [("bf16", 1, 1, 1, 128, 0), ("bf16", 37, 8, 2, 128, 1000000), ("bf16", 300, 32, 32, 64, 5),
                                                       ("fp32", 96, 4, 4, 64, 0), ("fp32", 5, 3, 1, 80, 2 ** 31 - 6), ("fp32", 2, 2, 2, 256, 77),
                                                       ("bf16", 3, 5, 3, 6, 9), ("fp32", 4, 1, 0, 2, 1), ("bf16", 2, 0, 2, 128, 4), ("bf16", 2000, 7, 1, 128, 3)])
def test_norm_rope(norm, dtype, rows, hq, hk, dh, start):
    b = _b()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k = _rand(33, rows, hq, dh, scale=3, dtype=dt), _rand(34, rows, hk, dh, scale=0.01, dtype=dt)
    if rows > 2 and hq:
        q[1] = 0
    pos = torch.arange(start, start + rows, dtype=torch.int64).clamp(max=2 ** 31 - 1).int()
    gq, gk = (_rand(35, dh, dtype=torch.float32) + 1, _rand(36, dh, dtype=torch.float32) + 1) if norm else (None, None)
    for inplace in (False, True):
        qi, ki = q.clone(), k.clone()
        qo, ko = b.qk_norm_rope(qi, ki, gq, gk, pos.to(DEV), theta=500000.0, eps=1e-5, q_out=qi if inplace else None, k_out=ki if inplace else None)
        for x, got, g in ((q, qo, gq), (k, ko, gk)):
            if not x.numel():
                continue
            want = plain.norm_rope(_np(x), None if g is None else _np(g), pos.numpy(), 500000.0, float(np.float32(1e-5)))
            # fp32 steps: the mean of dh squares (dh + 4 roundings, halved by the root), norm, gain, angle (2^-24 of a half turn, sine and cosine within 2 ulp), two
            # products and a sum: (dh / 2 + 16) 2^-24 of the pair's magnitude; then the store's half step
            pair = np.hypot(want[..., :dh // 2], want[..., dh // 2:])
            pair = np.concatenate((pair, pair), -1)
            tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + (dh / 2 + 16) * 2.0 ** -24 * pair
            assert (np.abs(_np(got) - want) <= tol).all(), float((np.abs(_np(got) - want) - tol).max())


def test_norm_rope_strides_alignment_and_default_positions():
    b = _b()
    wide = _rand(37, 11, 3, 4, 64)
    q, k = wide[:, 0], wide[:, 1]
    flat = _rand(38, 11 * 4 * 64 + 1)
    odd = flat[1:].view(11, 4, 64)                                      # rows not on 16 bytes
    odd.copy_(q)
    want, wk = b.qk_norm_rope(q.contiguous(), k.contiguous(), theta=100.0)
    got, gk = b.qk_norm_rope(q, k, theta=100.0)
    go, _ = b.qk_norm_rope(odd, k, theta=100.0)
    assert torch.equal(want, got) and torch.equal(wk, gk) and torch.equal(go, want)
    assert torch.equal(want, b.qk_norm_rope(q, k, positions=torch.arange(11, dtype=torch.int32, device=DEV), theta=100.0)[0])
    vcopy = wide[:, 2].clone()
    b.qk_norm_rope(q, k, theta=100.0, q_out=q, k_out=k)                 # in place inside the wide rows
    assert torch.equal(q, want) and torch.equal(k, wk) and torch.equal(wide[:, 2], vcopy)
    with pytest.raises(ValueError):
        b.qk_norm_rope(q, k.float())


# ---- together ----------------------------------------------------------------------------------------------------------------

def test_a_cached_decode_with_eviction():
    """Two sequences through norm + rotation, the cache, attention, weights and eviction, block after block, against the same in
    64 bits on what the cache holds."""
    b = _b()
    heads, group, dh, s, prompt, keep = 2, 2, 128, 16, 150, 120
    B, scale = 2, 128 ** -0.5
    cap = prompt + 3 * s
    c = b.KvCache4(B, heads, dh, cap)
    gain = _rand(40, dh, scale=0.1, dtype=torch.float32) + 1
    weights = torch.zeros(B, heads, cap, device=DEV)
    positions = torch.full((B, heads, cap), -1, dtype=torch.int32, device=DEV)
    lens = _i32([0, 0])
    mirror = [[([], [], []) for _ in range(heads)] for _ in range(B)]   # per head: keys, values, positions the cache holds
    seen = 0
    for step, rows in enumerate([prompt, s, s]):
        q, k, v = (_rand(50 + 3 * step + i, B, rows, h, dh) for i, h in enumerate((heads * group, heads, heads)))
        pos = torch.arange(seen, seen + rows, dtype=torch.int32, device=DEV).repeat(B)
        qr, kr = b.qk_norm_rope(q.view(B * rows, -1, dh), k.view(B * rows, heads, dh), gain, gain, pos, theta=10000.0)
        qr, kr = qr.view(q.shape), kr.view(k.shape)
        c.store(kr, v, key_start=lens)
        n0 = int(lens[0])
        positions[:, :, n0:n0 + rows] = torch.arange(seen, seen + rows, dtype=torch.int32, device=DEV)
        lens = lens + rows
        for i in range(B):
            for h in range(heads):
                mk, mv, mp = mirror[i][h]
                mk += list(plain.values(_np(kr[i, :, h]))); mv += list(plain.values(_np(v[i, :, h]))); mp += range(seen, seen + rows)
        seen += rows
        out, lse = c.attention(qr, lens, cap)
        before = weights.clone()
        c.attention_weights(qr, lse, lens, cap, weights)
        n = n0 + rows
        for i in range(B):
            for h in range(heads):
                mk, mv, mp = mirror[i][h]
                assert positions[i, h, :n].tolist() == list(mp)
                qh = _np(qr[i, :, h * group:(h + 1) * group])
                want, wl, ww = plain.attention(qh, np.array(mk)[:, None], np.array(mv)[:, None], scale)
                r = np.abs(mv).max()
                d = scale * (np.abs(qh).sum(-1).max() * 2 * np.abs(mk).max()) * 16 * 2.0 ** -23
                assert (np.abs(_np(out[i, :, h * group:(h + 1) * group]) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * d + 2.0 ** -18) * 2 * r).all()
                got = _np(weights[i, h, :n] - before[i, h, :n])
                assert np.abs(got - ww[0]).max() <= (2 * d + 2.0 ** -17) * max(1.0, ww.max(), float(weights[i, h, :n].max()))
        old = weights.double().cpu().numpy()
        kept, lens = c.evict(weights, lens, cap, keep, positions=positions, first=4, protect_from=_i32([seen - s] * B))
        for i in range(B):
            for h in range(heads):
                mk, mv, mp = mirror[i][h]
                want = plain.keep(old[i, h], list(mp), n, keep, 4, seen - s)
                assert kept[i, h, :len(want)].tolist() == want
                mirror[i][h] = ([mk[j] for j in want], [mv[j] for j in want], [mp[j] for j in want])
    assert lens.tolist() == [keep, keep]
